"""Page tables, windows, lengths and start orders against the documented steps, list by
list.  All results are whole numbers and have to be equal."""
from collections import deque

import pytest
import torch

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.page_tables import PageTables
from paper_2605_20600_amd.paged import PagedKV

pytestmark = pytest.mark.gpu


def _key(n):
    if n < 8:
        return max(n, 0)
    e = n.bit_length() - 1
    return (e - 2) * 8 + ((n >> (e - 3)) & 7)


def _oracle(t, advance, counts, tokens):
    """The state (dict of CPU tensors, changed in place) after a step."""
    layers, rows, ptok, num = t["layers"], t["rows"], t["ptok"], t["num"]
    pages, length, first = t["pages"], t["len"], t["first"]
    lists, heads, most = pages.shape
    state = t["free_state"].tolist()
    ring = t["free_pages"].tolist()
    places = [(state[0] + k) % num for k in range(state[1])]
    free = deque(ring[p] for p in places)
    end = (state[0] + state[1]) % num
    pg, ln, fs = pages.tolist(), length.tolist(), first.tolist()
    window = None if t["window"] is None else t["window"].tolist()

    def let_go(page):
        nonlocal end
        if len(free) < num:
            free.append(page)
            ring[end] = page
            end = (end + 1) % num

    n = [tokens if counts is None else min(max(int(counts[r]), 0), tokens) for r in range(rows)]
    for l in range(lists):
        gain = 0 if advance is None else int(advance[l % rows])
        for h in range(heads):
            before = max(fs[l][h], 0)
            if gain < 0:
                ln[l][h] = before = 0
                for p in range(most):
                    if 0 <= pg[l][h][p] < num:
                        let_go(pg[l][h][p])
                    pg[l][h][p] = -1
            else:
                ln[l][h] = min(max(ln[l][h], 0) + gain, most * ptok)
            fs[l][h] = before
            if window is not None and window[l][h] > 0:
                fs[l][h] = max(before, ln[l][h] + 1 - window[l][h])
            for p in range(before // ptok, min(fs[l][h] // ptok, most)):
                if 0 <= pg[l][h][p] < num:
                    let_go(pg[l][h][p])
                    pg[l][h][p] = -1
    head, lacks = state[0], 0
    for l in range(lists):
        for h in range(heads):
            for p in range(-(-ln[l][h] // ptok), min(-(-(ln[l][h] + n[l % rows]) // ptok), most)):
                if 0 <= pg[l][h][p] < num:
                    continue
                if free:
                    pg[l][h][p] = free.popleft()
                    head = (head + 1) % num
                else:
                    lacks += 1
    order = []
    for layer in range(layers):
        key = [_key(ln[l][h] + n[l % rows] - fs[l][h])
               for l in range(layer * rows, (layer + 1) * rows) for h in range(heads)]
        order.append(sorted(range(len(key)), key=lambda i: -key[i]))
    for name, x in (("pages", pg), ("len", ln), ("first", fs), ("order", order),
                    ("free_pages", ring), ("free_state", [head, len(free), lacks, 0])):
        t[name] = torch.tensor(x, dtype=torch.int32)


NAMES = ("pages", "len", "first", "order", "free_pages", "free_state")


def _state(tables, ptok):
    t = {name: getattr(tables, name).cpu().clone() for name in NAMES}
    t["window"] = None if tables.window is None else tables.window.cpu()
    return dict(t, rows=tables.rows, layers=tables.layers, ptok=ptok,
                num=tables.free_pages.numel())


def _same(tables, want):
    for name in NAMES:
        got = getattr(tables, name).cpu()
        assert torch.equal(got, want[name].view(got.shape)), name


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, dtype=torch.int32)


def _step(tables, want, tokens, advance=None, counts=None):
    tables.extend(tokens, advance=None if advance is None else advance.cuda(),
                  counts=None if counts is None else counts.cuda())
    _oracle(want, advance, counts, tokens)
    _same(tables, want)


@pytest.mark.parametrize("heads,rows,layers,ptok,most,windows", (
    (1, 1, 1, 32, 1, False), (3, 5, 1, 32, 9, True), (32, 8, 1, 64, 6, True),
    (20, 7, 4, 128, 5, False), (32, 64, 1, 32, 7, True), (8, 40, 8, 64, 9, True),
    (1, 3000, 2, 256, 2, False), (1024, 2, 3, 32, 4, True)))
def test_steps_of_a_generation(heads, rows, layers, ptok, most, windows):
    g = torch.Generator().manual_seed(heads + rows)
    lists = rows * layers
    window = None
    if windows:
        window = torch.where(torch.rand((lists, heads), generator=g) < 0.5,
                             _ints(g, 1, 2 * ptok, (lists, heads)), 0).to(torch.int32).cuda()
    tables = PageTables(heads, most, lists * heads * most + 3, rows, layers, page_tokens=ptok,
                        window=window)
    want = _state(tables, ptok)
    # prompts; drafted steps; rows that end and begin anew; one call for what is there already
    prompt = _ints(g, 0, ptok * most // 2 + 1, (rows,))
    _step(tables, want, int(prompt.max()), counts=prompt)
    advance = prompt
    for step in range(6):
        counts = _ints(g, -1, 6, (rows,))
        if step == 3:
            over = torch.rand(rows, generator=g) < 0.4
            advance = torch.where(over, -1 - step, advance).to(torch.int32)
            counts = torch.where(over, prompt, counts).to(torch.int32)
        _step(tables, want, max(5, int(prompt.max())), advance, counts)
        if step == 2:
            _step(tables, want, 5)
        advance = torch.minimum(counts.clamp(min=0), _ints(g, 0, 6, (rows,)))
    _step(tables, want, 0, torch.full((rows,), -1, dtype=torch.int32))
    assert int(tables.free_state[1]) == lists * heads * most + 3
    assert sorted(tables.free_pages.tolist()) == list(range(lists * heads * most + 3))


@pytest.mark.parametrize("rows,layers", ((6, 1), (300, 4)))
def test_too_few_pages(rows, layers):
    heads, most, g = 4, 8, torch.Generator().manual_seed(rows)
    num = rows * layers * heads * 2 + 1
    tables = PageTables(heads, most, num, rows, layers, page_tokens=32)
    want = _state(tables, 32)
    counts = _ints(g, 0, 150, (rows,))
    _step(tables, want, 150, counts=counts)
    assert int(tables.free_state[2]) > 0 and int(tables.free_state[1]) == 0
    # some end in the step in which others lack pages: theirs go on at once
    advance = torch.where(torch.rand(rows, generator=g) < 0.3, -1, 3).to(torch.int32)
    _step(tables, want, 150, advance, counts)
    _step(tables, want, 150, advance, counts)
    # lists past their tables
    _step(tables, want, 1 << 24, torch.full((rows,), 1 << 30, dtype=torch.int32))
    assert int(tables.len.max()) == 256


def test_what_a_table_should_not_hold():
    heads, rows, most, num = 2, 4, 6, 20
    tables = PageTables(heads, most, num, rows, page_tokens=32,
                        window=torch.tensor([[5, 0], [-3, 40], [1, 1], [0, 2 ** 31 - 1]],
                                            dtype=torch.int32).cuda())
    g = torch.Generator().manual_seed(1)
    # numbers that are none, pages twice, a ring of more than there are, lengths below 0
    tables.pages.copy_(_ints(g, -3, 24, (rows, heads, most)))
    tables.len.copy_(_ints(g, -5, 90, (rows, heads)))
    tables.first.copy_(_ints(g, -5, 60, (rows, heads)))
    tables.free_state.copy_(torch.tensor([19, 3, 7, 7]))
    want = _state(tables, 32)
    _step(tables, want, 40, torch.tensor([-1, 3, 50, 0], dtype=torch.int32),
          torch.tensor([40, -1, 12, 90], dtype=torch.int32))
    _step(tables, want, 3, torch.tensor([-1, -1, -1, -1], dtype=torch.int32))
    assert int(tables.free_state[1]) <= num


def test_as_many_lists_as_blocks_take_turns():
    # a block of 512 takes its lists 256 at a time
    heads, rows, most = 64, 9000, 2
    tables = PageTables(heads, most, rows * heads * 2, rows, page_tokens=32)
    want = _state(tables, 32)
    g = torch.Generator().manual_seed(2)
    counts = _ints(g, 0, 64, (rows,))
    _step(tables, want, 64, counts=counts)
    _step(tables, want, 3, torch.where(counts > 50, -1, counts).to(torch.int32))


def test_more_layers_than_blocks_sort():
    # 4096 blocks sort, one layer after the other
    tables = PageTables(1, 1, 20000, 2, 5000, page_tokens=32)
    want = _state(tables, 32)
    tables.len.copy_(_ints(torch.Generator().manual_seed(5), 0, 30, (10000, 1)))
    want["len"] = tables.len.cpu()
    _step(tables, want, 2, counts=torch.tensor([2, 1], dtype=torch.int32))


@pytest.mark.parametrize("rows,layers", ((8, 1), (64, 4)))
def test_replays_and_streams(rows, layers):
    heads, most = 16, 6
    g = torch.Generator().manual_seed(3)
    lists = rows * layers
    window = _ints(g, 0, 70, (lists, heads)).cuda()
    tables = PageTables(heads, most, lists * heads * most, rows, layers, page_tokens=32,
                        window=window)
    advance, counts = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    want = _state(tables, 32)
    side = torch.cuda.Stream()
    counts.fill_(40)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tables.extend(40, counts=counts)
    torch.cuda.current_stream().wait_stream(side)
    _oracle(want, None, counts.cpu(), 40)
    _same(tables, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tables.extend(9, advance=advance, counts=counts)
    _same(tables, want)
    for step in range(8):
        advance.copy_(_ints(g, -1 if step == 5 else 0, 9, (rows,)))
        counts.copy_(_ints(g, 0, 9, (rows,)))
        graph.replay()
        _oracle(want, advance.cpu(), counts.cpu(), 9)
        _same(tables, want)


def test_lists_that_calls_use():
    # tokens are written where the tables say, attended from where the windows begin
    heads, rows, layers, d = 4, 3, 2, 64
    window = torch.tensor([0, 40, 0, 7], dtype=torch.int32).repeat(rows * layers, 1).cuda()
    tables = PageTables(heads, 6, 200, rows, layers, page_tokens=32, window=window)
    cache = PagedKV("bf16", d, heads, 200, page_tokens=32)
    cache.pool.fill_(255)
    lists = [tables.lists(layer) for layer in range(layers)]
    g = torch.Generator().manual_seed(4)
    length = torch.zeros(rows, dtype=torch.int32)
    held = [torch.zeros((rows, 192, heads, d), dtype=torch.bfloat16) for _ in lists]
    for step in range(20):
        counts = _ints(g, 1, 9, (rows,))
        tables.extend(9, advance=advance.cuda() if step else None, counts=counts.cuda())
        for layer, l in enumerate(lists):
            k = torch.randn((rows, 9, heads, d), generator=g).to(torch.bfloat16)
            cache.write(l, k.cuda(), k.cuda(), counts=counts.cuda())
            for r in range(rows):
                at, n = int(length[r]), int(counts[r])
                held[layer][r, at:at + n] = k[r, :n]
        advance = torch.minimum(counts, _ints(g, 0, 9, (rows,)))
        length += advance
    tables.extend(0, advance=advance.cuda())
    assert torch.equal(tables.len.cpu()[:rows, 0], length)
    for layer, l in enumerate(lists):
        k, v = cache.read(l, 192)
        for r in range(rows):
            for h, w in enumerate((0, 40, 0, 7)):
                lo, n = max(0, int(length[r]) + 1 - w) if w else 0, int(length[r])
                assert torch.equal(k[r, lo:n, h].cpu(), held[layer][r, lo:n, h])
                assert torch.equal(v[r, lo:n, h].cpu(), held[layer][r, lo:n, h])
                assert bool((k[r, n:, h] == 0).all())


def test_refusals():
    tables = PageTables(4, 2, 10, 3, 2)
    ok = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in (dict(advance=ok.long()), dict(counts=ok[:2]), dict(advance=ok.cpu())):
        with pytest.raises(ValueError):
            tables.extend(1, **kw)
    with pytest.raises(ValueError):
        tables.lists(2)
    with pytest.raises(ValueError):
        PageTables(4, 2, 10, 3, 2, window=ok)
    for kw in (dict(tokens=-1), dict(tokens=1 << 25)):
        with pytest.raises(B.HeadKVError):
            tables.extend(**kw)
    with pytest.raises(B.HeadKVError):
        PageTables(4, 2, 10, 3, page_tokens=48)
    with pytest.raises(ValueError):  # of another cache
        PagedKV("int8", 64, 8, 10)._check_lists(tables.lists())
