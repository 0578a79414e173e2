"""The paged cache (write, read) and attention over it against plain 64-bit
implementations of the formulas in headkv.h.

What is written and read back has one right answer, bit for bit.  Attention is
held to a bound on fp32 arithmetic, from the data (u = 2^-23, one rounding or
two): a score sums d products, |ds| <= (d + 4) u sum |q_i k_i| / sqrt(d); the
exponential adds 2^-20 (its argument, rounded, and its own error) and |s| u;
so each weight is off by at most e = 2 ds + 2^-20 + 2 |s|max u relatively, the
weighted mean of n values of at most vmax by 2 (e + (n + 8) u) vmax, and the log
of the sum by e + (n + 8) u + |lse| u.

Every pool is filled with bytes 255 first (NaN as bf16 and as any scale), so
that what was never written may not be seen.
"""
import math

import pytest
import torch

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.paged import PagedKV

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
TYPES = ("bf16", "int8", "fp4")
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def _held(x, kind):
    """What a cache holds for x [..., d] (bf16, CPU), in 64 bits."""
    x = x.double()
    if kind == "bf16":
        return x
    if kind == "int8":
        top = x.abs().amax(-1, keepdim=True)
        s = (top / 127).to(torch.bfloat16).double()
        n = torch.where(s > 0, x / s, torch.zeros_like(x)).round().clamp(-127, 127)
        return torch.where(top.isfinite(), n * s, torch.full_like(x, math.nan))
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -126)
    for p in range(-126, 127):  # the smallest power that is large enough
        e = torch.where((e == p) & (top > 6 * 2.0 ** p), p + 1.0, e)
    a = y.abs() / 2.0 ** e
    i = torch.zeros(a.shape, dtype=torch.long)
    for j in range(7):
        mid = (GRID[j] + GRID[j + 1]) / 2
        i = torch.where((a > mid) | ((a == mid) & (j % 2 == 1)), j + 1, i)
    v = GRID[i] * 2.0 ** e * torch.sign(y)
    return torch.where(top.isfinite(), v, torch.full_like(y, math.nan)).reshape(x.shape)


def _cache(kind, d, heads, num_pages, **kw):
    c = PagedKV(kind, d, heads, num_pages, **kw)
    c.pool.fill_(255)
    return c


def _table(lists, heads, pages, num_pages, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(num_pages, generator=g)[:lists * heads * pages].to(torch.int32).view(
        lists, heads, pages).cuda()


def _values(shape, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1] + (1,),
                                                                         generator=g))
    return x.to(torch.bfloat16)


def _same(got, want):
    got, want = got.cpu(), want.to(torch.bfloat16)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(0), want.nan_to_num(0)), \
        float((got.double() - want.double()).abs().nan_to_num(0).max())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("ptok", (32, 256))
def test_written_and_read_back(kind, d, ptok):
    # lists that grow in steps of odd sizes, from lengths inside a block of eight
    lists, heads, most = 3, 5, 2 * ptok + 40
    c = _cache(kind, d, heads, 200, page_tokens=ptok)
    table = _table(lists, heads, -(-most // ptok), 200, 1)
    start = torch.tensor([[0, 1, 7, 8, 9], [31, 32, 33, ptok - 1, ptok], [3, 5, 2, 4, 6]],
                         dtype=torch.int32).cuda()
    l = c.lists(table, start, max_len=int(start.max()))
    done = 0
    want_k, want_v, got = [], [], []
    for i, tokens in enumerate((1, 1, 2, 5, 8, 1, 17)):
        k, v = (_values((lists, tokens, heads, d), 10 * i + j) for j in range(2))
        c.write(l, k.cuda(), v.cuda())
        l.advance(tokens)
        done += tokens
        want_k.append(_held(k, kind))
        want_v.append(_held(v, kind))
    k, v = c.read(l, done, begin=-done)
    _same(k, torch.cat(want_k, 1))
    _same(v, torch.cat(want_v, 1))
    # the tokens past the end are zeros, and so is what lies before the first
    k, v = c.read(l, 3, begin=most - 3)
    assert not k.any() and not v.any()
    k, v = c.read(c.lists(table, None, max_len=0), 5, begin=-2)
    assert not k.any() and not v.any()


@pytest.mark.parametrize("kind", TYPES)
def test_rounding_edges(kind):
    # ties in both directions, rows of zeros, of the smallest and largest numbers,
    # infinities and NaN
    d = 64
    rows = [torch.zeros(d)]
    i = torch.arange(d)
    rows.append((i - 32).float())                     # ties of int8 at half the scale
    rows.append(torch.where(i % 2 == 0, 127.0, 63.5 - i))
    rows.append(torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 8))
    rows.append(-torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 8) * 2.0 ** 20)
    rows.append(torch.tensor([6.0, 6.03125, 0.5, 0.52, 0.49, 3.0, 12.0, 1.0] * 8))
    rows.append((i - 20).float() * 2.0 ** -133)       # subnormal numbers
    rows.append((i - 31).float() * 2.0 ** -120)
    rows.append(torch.full((d,), 3.3895313892515355e38) * torch.where(i % 3 == 0, -1.0, 0.4))
    rows.append(torch.where(i == 5, math.inf, 1.0))
    rows.append(torch.where(i == 40, -math.inf, 1.0))
    rows.append(torch.where(i == 63, math.nan, 1.0))
    rows.append(torch.where(i == 0, -math.nan, -2.0))
    x = torch.stack(rows).to(torch.bfloat16)[None, :, None]
    g = torch.Generator().manual_seed(3)
    many = torch.randint(0, 65536, (1, 4000, 1, d), generator=g).to(torch.int32).to(torch.int16)
    bits = many.view(torch.bfloat16)
    for x in (x, torch.where(bits.isfinite(), bits, torch.ones_like(bits))):
        n = x.shape[1]
        c = _cache(kind, d, 1, 80)
        l = c.lists(_table(1, 1, 70, 80, 2), None, max_len=0)
        c.write(l, x.cuda(), x.flip(1).contiguous().cuda())
        l.advance(n)
        k, v = c.read(l, n)
        _same(k, _held(x, kind))
        _same(v, _held(x.flip(1), kind))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("tokens", (1, 4))
def test_rounding_of_few_tokens(kind, d, tokens):
    # any bits, infinities and NaN among them, and rows of small numbers only
    lists, heads = 300, 3
    g = torch.Generator().manual_seed(d + tokens)
    for scale in (0, 2.0 ** -130):
        x = torch.randint(0, 65536, (2, lists, tokens, heads, d), generator=g).to(torch.int32)
        x = x.to(torch.int16).view(torch.bfloat16)
        if scale:
            x = (torch.randn(x.shape, generator=g) * scale).to(torch.bfloat16)
        else:  # every other row without infinities and NaN
            x[:, ::2] = torch.where(x[:, ::2].isfinite(), x[:, ::2], torch.ones_like(x[:, ::2]))
        c = _cache(kind, d, heads, lists * heads)
        l = c.lists(_table(lists, heads, 1, lists * heads, 2), None, max_len=0)
        c.write(l, x[0].cuda(), x[1].cuda())
        l.advance(tokens)
        k, v = c.read(l, tokens)
        _same(k, _held(x[0], kind))
        _same(v, _held(x[1], kind))


@pytest.mark.parametrize("kind", TYPES)
def test_strides_counts_dropped_pages_and_bounds(kind):
    lists, heads, d, tokens = 4, 3, 128, 90
    c = _cache(kind, d, heads, 64, page_tokens=32)
    before = c.pool.clone()
    table = _table(lists, heads, 3, 64, 4)
    table[1, 2, 1] = -1
    table[2, 0, 0] = 64  # not a page of the pool
    # k and v inside a packed projection, heads first
    packed = _values((lists, heads, tokens, 3 * d), 7).cuda()
    k, v = (packed[..., i * d:(i + 1) * d].transpose(1, 2) for i in (1, 2))
    counts = torch.tensor([90, 0, 33, 1000], dtype=torch.int32).cuda()
    l = c.lists(table, torch.zeros((lists, heads), dtype=torch.int32, device="cuda"), max_len=6,
                extra=6)
    c.write(l, k, v, counts)
    l.advance(90)
    got = c.read(l, 90, begin=6)
    there = torch.zeros((lists, 90, heads, 1), dtype=torch.bool)
    for i, n in enumerate((90, 0, 33, 90)):
        there[i, :n] = True
    at = torch.arange(90) + 6
    there[1, :, 2] &= ~((at >= 32) & (at < 64))[:, None]
    there[2, :, 0] &= (at >= 32)[:, None]
    for x, y in zip(got, (k, v)):
        want = _held(y.cpu(), kind)
        have = there.expand_as(want)
        _same(torch.where(have, x.cpu(), 0), torch.where(have, want, 0))
    # dropped pages read as zeros, not as what lies in the pool
    assert not got[0][1, 26:58, 2].any() and not got[1][2, :26, 0].any()
    # no byte of another page has changed
    used = set(table.flatten().tolist())
    pb = c.page_bytes
    for p in range(64):
        if p not in used:
            assert torch.equal(c.pool[p * pb:(p + 1) * pb], before[p * pb:(p + 1) * pb])
    # past the table's end nothing is stored
    full = c.pool.clone()
    l = c.lists(table, None, max_len=0, extra=96)
    c.write(l, k, v)
    assert torch.equal(c.pool, full)


def _reference(q, k, v, seen):
    """q [heads][group][d], k, v [tokens][heads][d] in 64 bits, seen [heads][tokens]:
    out, lse and the bounds of their errors."""
    d = q.shape[-1]
    s = torch.einsum("hgd,thd->hgt", q, k) / math.sqrt(d)
    mag = torch.einsum("hgd,thd->hgt", q.abs(), k.abs()) / math.sqrt(d)
    gone = ~seen[:, None].expand_as(s)
    s = s.masked_fill(gone, -math.inf)
    lse = torch.logsumexp(s, -1) if s.shape[-1] else s.new_full(s.shape[:2], -math.inf)
    w = torch.softmax(s, -1).nan_to_num(0.0)
    out = torch.einsum("hgt,thd->hgd", w, v)
    n = seen.sum(-1).max() if seen.numel() else 0
    ds = (d + 4) * U * float(mag.masked_fill(gone, 0).max() if mag.numel() else 0)
    smax = float(s.masked_fill(gone, 0).abs().max()) if s.numel() else 0.0
    e = 2 * ds + 2.0 ** -20 + 2 * smax * U
    vmax = float((v.abs() * seen.T[..., None]).max()) if v.numel() else 0.0
    return out, lse, 2 * (e + (n + 8) * U) * vmax, e + (n + 8) * U


class Setup:
    """Lists of given lengths with their contents kept in 64 bits."""

    def __init__(self, kind, d, heads, lens, ptok=64, group=1, prefix_lens=None, seed=0,
                 num_pages=None, page_base=0):
        lens = torch.tensor(lens, dtype=torch.int32)
        self.kind, self.group = kind, group
        sets = [lens] + ([] if prefix_lens is None else
                         [torch.tensor(prefix_lens, dtype=torch.int32)])
        per = [max(1, -(-int(x.max()) // ptok)) + 1 for x in sets]
        need = sum(x.numel() * p for x, p in zip(sets, per))
        self.c = _cache(kind, d, heads, (num_pages or need + 5), page_tokens=ptok, group=group)
        g = torch.Generator().manual_seed(seed)
        perm = (torch.randperm(need, generator=g) + page_base).to(torch.int32)
        self.lists, self.k, self.v, self.lens = [], [], [], sets
        at = 0
        for i, (x, p) in enumerate(zip(sets, per)):
            table = perm[at:at + x.numel() * p].view(*x.shape, p).cuda()
            at += x.numel() * p
            most = max(1, int(x.max()))
            k = _values((x.shape[0], most, heads, d), seed + 2 * i + 1, 0.7)
            v = _values((x.shape[0], most, heads, d), seed + 2 * i + 2, 0.7)
            zero = torch.zeros_like(x).cuda()
            self.c.write(self.c.lists(table, zero, max_len=0), k.cuda(), v.cuda())
            # what lies past the length goes back to bytes 255, as if never written
            l = self.c.lists(table, x.cuda(), max_len=int(x.max()))
            self.lists.append(l)
            self.k.append(_held(k, kind))
            self.v.append(_held(v, kind))
        g2 = torch.Generator().manual_seed(seed + 77)
        self.q = (1.3 * torch.randn((lens.shape[0], heads * group, d), generator=g2)).to(
            torch.bfloat16)

    def check(self, first=None, share=None, dropped=(), max_len=None, q=None, q_dev=None,
              shared_first=None, shared_dropped=()):
        own = self.lists[0]
        own.arg.max_len = own.arg.max_len if max_len is None else max_len
        keep = []
        if first is not None:
            keep.append(torch.tensor(first, dtype=torch.int32).cuda())
            own.arg.first = keep[-1].data_ptr()
        if shared_first is not None:
            keep.append(torch.tensor(shared_first, dtype=torch.int32).cuda())
            self.lists[1].arg.first = keep[-1].data_ptr()
        q = self.q if q is None else q
        q_dev = q.cuda() if q_dev is None else q_dev
        bsz, hq, d = q.shape
        heads = hq // self.group
        out = torch.full((bsz, hq, d), math.nan, device="cuda")
        lse = torch.full((bsz, hq), math.nan, device="cuda")
        kw = {}
        if share is not None:
            kw = dict(shared=self.lists[1], share=torch.tensor(share, dtype=torch.int32).cuda())
        for again in range(2):  # the workspace is left as it was found
            self.c.attn(own, q_dev, out=out, lse=lse, **kw)
            torch.cuda.synchronize()
            if again:
                assert torch.equal(out.nan_to_num(7), last.nan_to_num(7)), "not deterministic"
            last = out.clone()
        got, got_lse = out.cpu().double(), lse.cpu().double()
        for b in range(bsz):
            k, v = self.k[0][b], self.v[0][b]
            t = torch.arange(k.shape[0])
            n = self.lens[0][b].clone().clamp(max=own.arg.max_len)
            seen = t[None] < n[:, None]
            if first is not None:
                seen &= t[None] >= torch.tensor(first)[b][:, None]
            for (db, dh, dp) in dropped:
                if db == b:
                    ptok = self.c.cfg.page_tokens
                    seen[dh, dp * ptok:(dp + 1) * ptok] = False
            if share is not None and 0 <= share[b] < self.k[1].shape[0]:
                j = share[b]
                pk, pv = self.k[1][j], self.v[1][j]
                at = torch.arange(pk.shape[0])
                ps = at[None] < self.lens[1][j][:, None]
                if shared_first is not None:
                    ps &= at[None] >= torch.tensor(shared_first)[j][:, None]
                for (db, dh, dp) in shared_dropped:
                    if db == j:
                        ps[dh, dp * self.c.cfg.page_tokens:(dp + 1) * self.c.cfg.page_tokens] = False
                k, v, seen = torch.cat((pk, k)), torch.cat((pv, v)), torch.cat((ps, seen), 1)
            ref, ref_lse, tol, tol_lse = _reference(
                q[b].double().view(heads, self.group, d), k, v, seen)
            ref, ref_lse = ref.reshape(hq, d), ref_lse.reshape(hq)
            err = float((got[b] - ref).abs().max())
            assert err <= tol, (b, err, tol)
            empty = ref_lse == -math.inf
            assert torch.equal(got_lse[b] == -math.inf, empty)
            assert not got[b][empty].any()
            d_lse = (got_lse[b] - ref_lse)[~empty].abs()
            assert bool((d_lse <= tol_lse + ref_lse[~empty].abs() * U).all()), (b, d_lse.max())


LENS = [[0, 1, 31, 32], [33, 63, 64, 65], [200, 127, 3, 0], [96, 95, 300, 129]]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("group", (1, 3, 16))
def test_attention_of_ragged_lists(kind, d, group):
    Setup(kind, d, 4, LENS, group=group, seed=d + group).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ptok", (32, 128, 256))
def test_attention_windows_and_dropped_pages(kind, ptok):
    s = Setup(kind, 128, 4, [[700, 513, 512, 511], [40, 700, 1, 650]], ptok=ptok, group=2, seed=5)
    first = [[0, 500, 512, 100], [39, 650, 1, 31]]  # [1][2] is left empty
    dropped = [(0, 0, 1), (1, 3, 0), (1, 1, 600 // ptok)]
    for i, (b, h, p) in enumerate(dropped):
        s.lists[0].pages[b, h, p] = (-1, s.c.cfg.num_pages, -7)[i]
    s.check(first=first, dropped=dropped)


@pytest.mark.parametrize("kind", TYPES)
def test_attention_of_lists_all_empty(kind):
    s = Setup(kind, 64, 2, [[0, 0], [0, 0]])
    s.check()
    s = Setup(kind, 64, 2, [[50, 9], [70, 1]])
    s.check(first=[[50, 10], [2 ** 31 - 1, 1]])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group,rows", ((1, 5), (1, 40), (4, 37), (7, 11), (16, 20)))
def test_attention_with_shared_prefixes(kind, group, rows):
    # rows in turn share lists 0, 2, none (-1, 3 = no such list) and the empty list 1
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 130, (rows, 2), generator=g).tolist()
    s = Setup(kind, 128, 2, lens, group=group, prefix_lens=[[333, 64], [0, 0], [31, 1025]],
              seed=group)
    s.check(share=[(0, 2, 0, -1, 1, 0, 3)[i % 7] for i in range(rows)])
    s.check(share=[0] * rows)
    s.check(share=[-1] * rows)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,ptok,group,rows", ((128, 64, 16, 43), (64, 32, 7, 60), (128, 256, 2, 131),
                                              (64, 64, 13, 41)))
def test_prefixes_of_many_columns(kind, d, ptok, group, rows):
    # windows that start and pages that are dropped inside a chunk, chunks past the
    # first, an own list that is empty, one list with nearly all columns
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 60, (rows, 2), generator=g).tolist()
    s = Setup(kind, d, 2, lens, ptok=ptok, group=group, prefix_lens=[[4400, 97], [290, 0]], seed=d)
    share = [(0, 0, 1, -1, 0)[i % 5] for i in range(rows)]
    s.check(share=share)
    s.check(share=[0] * (rows - 1) + [1])
    for i, (b, h, p) in enumerate(((0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1))):
        s.lists[1].pages[b, h, p] = (-1, s.c.cfg.num_pages, -7)[i]
    s.check(share=share, shared_first=[[1003, 96], [31, 5]],
            shared_dropped=[(0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1)])


@pytest.mark.parametrize("kind", TYPES)
def test_prefix_windows_and_dropped_pages(kind):
    s = Setup(kind, 128, 2, [[3, 40]] * 9, group=3, prefix_lens=[[700, 97], [290, 0]], seed=6)
    for i, (b, h, p) in enumerate(((0, 0, 2), (0, 1, 0), (1, 0, 1))):
        s.lists[1].pages[b, h, p] = (-1, s.c.cfg.num_pages, -7)[i]
    s.check(share=[0, 1, 0, 0, 1, -1, 0, 0, 0], shared_first=[[130, 96], [2 ** 31 - 1, 5]],
            shared_dropped=[(0, 0, 2), (0, 1, 0), (1, 0, 1)])


@pytest.mark.parametrize("d", (64, 128))
def test_attention_with_a_shared_prefix_and_nothing_else(d):
    s = Setup("int8", d, 3, [[0, 0, 0]] * 9, prefix_lens=[[1, 40, 2500]], seed=9)
    s.check(share=[0] * 8 + [-1])


@pytest.mark.parametrize("kind", TYPES)
def test_attention_of_long_lists(kind):
    Setup(kind, 128, 1, [[9001], [8192], [17]], group=2, seed=11).check()
    Setup(kind, 64, 1, [[16384]], group=1, prefix_lens=[[6000]], seed=12).check(share=[0])


def test_lengths_past_the_bound_and_extra():
    s = Setup("int8", 128, 2, [[100, 300], [257, 20]])
    s.check(max_len=130)  # tokens past max_len are not attended
    s = Setup("int8", 128, 2, [[100, 300], [257, 20]])
    l = s.lists[0]
    shorter = (s.lens[0] - 9).cuda()  # counted on the host instead
    l.arg.len, l.arg.extra = shorter.data_ptr(), 9
    s.check()
    negative = torch.full((2, 2), -2 ** 31, dtype=torch.int32, device="cuda")
    l.arg.len, l.arg.extra = negative.data_ptr(), 0
    s.lens[0] = torch.zeros((2, 2), dtype=torch.int32)
    s.check()
    most = torch.full((2, 2), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    l.arg.len, l.arg.extra, l.arg.max_len = most.data_ptr(), 2 ** 31 - 1, 20
    s.lens[0] = torch.full((2, 2), 20, dtype=torch.int32)
    s.check()


def test_queries_of_any_stride():
    s = Setup("fp4", 64, 3, [[70, 1, 200]] * 5, group=2)
    wide = torch.full((5, 3 * 6 * 64), math.nan, dtype=torch.bfloat16, device="cuda")
    q_dev = wide[:, 128:128 + 6 * 64].view(5, 6, 64)
    q_dev.copy_(s.q)
    assert q_dev.stride(0) == 3 * 6 * 64
    s.check(q_dev=q_dev)
    same = s.q[:1].expand(5, 6, 64)  # one query for all rows
    s.check(q=same, q_dev=same[:1].cuda().expand(5, 6, 64))


@pytest.mark.parametrize("kind", TYPES)
def test_large_scores(kind):
    s = Setup(kind, 128, 2, [[400, 65], [33, 130]], seed=21)
    s.q = (s.q.float() * 300).to(torch.bfloat16)
    s.check()


@pytest.mark.parametrize("kind", TYPES)
def test_pages_past_four_gigabytes(kind):
    page = {"bf16": 131072, "int8": 66560, "fp4": 34816}[kind]
    base = (1 << 32) // page + 7
    s = Setup(kind, 128, 2, [[300, 513], [64, 1]], ptok=256, num_pages=base + 60, page_base=base,
              prefix_lens=[[700, 30]])
    assert s.c.pool.numel() > 1 << 32
    s.check(share=[0, 0])
    k, v = s.c.read(s.lists[0], 513)
    for b in range(2):
        for h, n in enumerate(s.lens[0][b].tolist()):
            _same(k[b, :n, h], s.k[0][b, :n, h])
            _same(v[b, :n, h], s.v[0][b, :n, h])


@pytest.mark.parametrize("kind", TYPES)
def test_a_nan_stays_in_its_head(kind):
    s = Setup(kind, 128, 3, [[200, 200, 200]], seed=31)
    clean = s.c.attn(s.lists[0], s.q.cuda()).clone()
    k = torch.ones((1, 1, 3, 128), dtype=torch.bfloat16)
    k[0, 0, 1, 77] = math.nan
    at = s.c.lists(s.lists[0].pages, None, max_len=0, extra=130)
    k_old, v_old = s.c.read(at, 1, begin=130)
    k_all, v_all = s.c.read(s.lists[0], 200)
    k_new = k_all[:, 130:131].clone()
    k_new[0, 0, 1] = k[0, 0, 1].cuda()
    s.c.write(at, k_new, v_all[:, 130:131].contiguous())
    got = s.c.attn(s.lists[0], s.q.cuda())
    assert got[0, 1].isnan().all()
    # the other heads' rows were written again from their own values
    assert got[0, 0].isfinite().all() and got[0, 2].isfinite().all()
    if kind == "bf16":
        assert torch.equal(got[0, 0], clean[0, 0]) and torch.equal(got[0, 2], clean[0, 2])


def test_calls_of_any_sizes_share_the_workspace():
    setups = [Setup("int8", 128, 2, torch.randint(1, n, (rows, 2), generator=torch.Generator()
                                                  .manual_seed(rows)).tolist(), group=group, seed=rows)
              for rows, n, group in ((3, 3000, 1), (200, 40, 2), (2, 5000, 16), (60, 1200, 1))]
    ws = max((s.c._workspace(s.lists[0], None) for s in setups), key=lambda t: t.numel())
    for s in setups * 2:
        s.c._ws = ws
        s.check()


def test_more_lists_than_counters():
    # 660 x 100 lists of up to two tokens, and eight rows with longer ones that are cut
    batch, heads, d, ptok, most = 660, 100, 64, 32, 1300
    rows = [0, 1, 97, 500, 654, 655, 656, 659]
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 3, (batch, heads), generator=g).to(torch.int32)
    lens[rows, ::3] = torch.randint(1100, most, (len(rows), 34), generator=g).to(torch.int32)
    per = -(-most // ptok)
    table = torch.full((batch, heads, per), -1, dtype=torch.int32)
    need = (lens + ptok - 1) // ptok
    there = torch.arange(per) < need[..., None]
    n = int(there.sum())
    table[there] = torch.randperm(n, generator=g).to(torch.int32)
    c = _cache("fp4", d, heads, n, page_tokens=ptok)
    k, v = (_values((len(rows), most, heads, d), i, 0.7) for i in range(2))
    c.write(c.lists(table[rows].contiguous().cuda(), None, max_len=0), k.cuda(), v.cuda())
    rest = [b for b in range(batch) if b not in rows]
    kr, vr = (_values((len(rest), 2, heads, d), 3 + i, 0.7) for i in range(2))
    c.write(c.lists(table[rest].contiguous().cuda(), None, max_len=0), kr.cuda(), vr.cuda())
    q = _values((batch, heads, d), 7, 0.3)
    for order in (True, False):
        l = c.lists(table.cuda(), lens.cuda(), max_len=most)
        if not order:
            l.arg.order = None
        got = c.attn(l, q.cuda()).cpu().double()
        for i, b in enumerate(rows + rest[::50]):
            kb, vb = (k[i], v[i]) if b in rows else (kr[rest.index(b)], vr[rest.index(b)])
            kb, vb = _held(kb, "fp4"), _held(vb, "fp4")
            seen = torch.arange(kb.shape[0])[None] < lens[b][:, None]
            ref, _, tol, _ = _reference(q[b].double().view(heads, 1, d), kb, vb, seen)
            assert float((got[b] - ref[:, 0]).abs().max()) <= tol, b


def test_on_another_stream():
    s = Setup("int8", 128, 4, LENS, seed=41)
    want = s.c.attn(s.lists[0], s.q.cuda()).clone()
    q = s.q.cuda()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = s.c.attn(s.lists[0], q)
    st.synchronize()
    assert torch.equal(got, want)


def test_in_a_graph():
    s = Setup("int8", 128, 4, LENS, prefix_lens=[[100, 1, 64, 333]], seed=43)
    q = s.q.cuda()
    share = torch.tensor([0, 0, -1, 0], dtype=torch.int32).cuda()
    out = torch.empty((4, 4, 128), device="cuda")
    k = _values((4, 1, 4, 128), 5).cuda()
    l = s.c.lists(s.lists[0].pages, s.lists[0].length, max_len=301)
    grown = s.c.lists(s.lists[0].pages, s.lists[0].length, max_len=301, extra=1)

    def step():
        s.c.write(l, k, k)
        s.c.attn(grown, q, shared=s.lists[1], share=share, out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        k.copy_(_values((4, 1, 4, 128), 100 + i))
        q.copy_(s.q * (1 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out), i


def test_python_refusals():
    c = PagedKV("int8", 128, 2, 10)
    pages = torch.zeros((1, 2, 3), dtype=torch.int32, device="cuda")
    l = c.lists(pages, None, max_len=0)
    good = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        c.lists(pages.long(), None, max_len=0)
    with pytest.raises(ValueError):
        c.lists(pages[:, :1].contiguous(), None, max_len=0)
    with pytest.raises(ValueError):
        c.write(l, good.float(), good.float())
    with pytest.raises(ValueError):
        c.write(l, good, good.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        c.write(l, good, good, counts=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        c.read(l, 3, k=good, v=good)
    with pytest.raises(ValueError):
        c.attn(l, good[:, 0].float())
    with pytest.raises(B.HeadKVError) as e:
        c.attn(l, good[:, 0], shared=l)
    assert e.value.status == B.HEADKV_ERR_INVALID_ARG


def test_python_refuses_other_heads_and_host_memory():
    c = PagedKV("int8", 128, 2, 10)
    pages = torch.zeros((1, 1, 3), dtype=torch.int32, device="cuda")
    other = PagedKV("int8", 128, 1, 10).lists(pages, None, max_len=0)
    own = c.lists(pages.expand(1, 2, 3).contiguous(), None, max_len=0)
    rows = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16, device="cuda")
    share = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        c.write(other, rows, rows)
    with pytest.raises(ValueError):
        c.read(other, 4)
    with pytest.raises(ValueError):
        c.attn(other, rows[:, 0])
    with pytest.raises(ValueError):
        c.attn(own, rows[:, 0], shared=other, share=share)
    with pytest.raises(ValueError):
        c.lists(own.pages.cpu(), None, max_len=0)
    with pytest.raises(ValueError):
        c.write(own, rows.cpu(), rows.cpu())
    with pytest.raises(ValueError):
        c.write(own, rows, rows, counts=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        c.attn(own, rows[:, 0].cpu())
    with pytest.raises(ValueError):
        c.attn(own, rows[:, 0], out=torch.zeros((1, 2, 128)))
    with pytest.raises(ValueError):
        c.attn(own, rows[:, 0], lse=torch.zeros((1, 2)))
    with pytest.raises(ValueError):
        c.attn(own, rows[:, 0], shared=own, share=share.cpu())


def test_lists_shorter_than_the_tables():
    # 20 x 5 lists in tables of 21 pages of 64: 1280 tokens take more chunks than 1344
    g = torch.Generator().manual_seed(3)
    table = torch.randperm(2100, generator=g).to(torch.int32).view(20, 5, 21).cuda()
    c = _cache("int8", 64, 5, 2100)
    k, v = (torch.randn((20, 1280, 5, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    c.write(c.lists(table, None, max_len=0), k, v)
    q = torch.randn((20, 5, 64), generator=g).to(torch.bfloat16).cuda()
    n = torch.full((20, 5), 1280, dtype=torch.int32).cuda()
    a = c.attn(c.lists(table, n, max_len=1280), q)
    b = c.attn(c.lists(table, n, max_len=1344), q)
    # other chunks, the same sums: 1280 weighted values of less than 6, added in another order
    assert float((a - b).abs().max()) <= 2 * 1280 * U * 6


def test_first_use_in_a_graph():
    # the workspace that a capture makes belongs to the graph alone
    s = Setup("fp4", 64, 2, [[700, 3], [1, 900], [64, 500]], seed=47)
    q = s.q.cuda()
    want = s.c.attn(s.lists[0], q).clone()
    fresh = PagedKV("fp4", 64, 2, s.c.cfg.num_pages, page_tokens=s.c.cfg.page_tokens)
    fresh.pool.copy_(s.c.pool)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = fresh.attn(s.lists[0], q)
    eager = fresh.attn(s.lists[0], q)  # before any replay
    assert torch.equal(eager, want)
    for _ in range(3):
        captured.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, want)
        assert torch.equal(fresh.attn(s.lists[0], q), want)


def _short_lists(rows, heads, most, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, most + 1, (rows, heads), generator=g)
    lens[0, 0], lens[-1, -1], lens[1] = most, 0, 0  # a row without tokens
    return lens.tolist()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group", ((64, 1), (64, 5), (128, 1), (128, 16)))
def test_many_short_lists(kind, d, group):
    # 60 x 16 lists of up to 100 tokens: a wavefront each
    s = Setup(kind, d, 16, _short_lists(60, 16, 100, d + group), ptok=32, group=group, seed=51)
    s.check()
    first = torch.randint(-3, 110, (60, 16), generator=torch.Generator().manual_seed(1))
    first[2] = 2 ** 31 - 1
    s.check(first=first.tolist())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group", (1, 3, 7))
def test_many_short_lists_with_shared_prefixes(kind, group):
    # in the order of the launch, rows of two prefixes, of one without tokens and of none
    g = torch.Generator().manual_seed(group)
    rows = 16 if group > 1 else 40
    heads = 50
    prefix = torch.randint(0, 1400, (3, heads), generator=g)
    prefix[2] = 0
    s = Setup(kind, 64, heads, _short_lists(rows, heads, 80, 9), group=group, seed=53,
              prefix_lens=prefix.tolist())
    share = torch.randint(-1, 4, (rows,), generator=g).tolist()  # (3 is no list)
    share[0], share[1] = 0, 0
    s.check(share=share)
    first = torch.randint(0, 60, (rows, heads), generator=g).tolist()
    s.check(share=share, first=first)
    s.check(share=[1] * rows, first=first,
            shared_first=torch.randint(0, 900, (3, heads), generator=g).tolist())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group", (1, 5, 16))
def test_prefixes_and_long_lists_in_one_launch(kind, group):
    # both in several parts, rows that end in the middle of a column tile
    s = Setup(kind, 128, 2, [[1500, 0], [3, 700], [0, 0], [900, 2100], [64, 1]], group=group, seed=57,
              prefix_lens=[[1700, 1], [30, 2500]])
    s.check(share=[0, 1, 0, 1, 1])
    s.check(share=[0, 0, 0, 0, 0], first=[[1400, 0], [0, 650], [0, 0], [899, 3], [64, 0]])


def test_shared_prefix_and_more_lists_than_counters():
    # the shared lists' launch cannot join the rows' own: 66000 of them
    batch, heads, d, ptok = 660, 100, 64, 32
    g = torch.Generator().manual_seed(15)
    lens = torch.randint(0, 60, (batch, heads), generator=g).to(torch.int32)
    # all rows read the same two pages of a head, each as many tokens as it has
    table = torch.arange(2 * heads, dtype=torch.int32).view(1, heads, 2)
    prefix = torch.arange(2 * heads, 5 * heads, dtype=torch.int32).view(1, heads, 3)
    c = _cache("int8", d, heads, 5 * heads, page_tokens=ptok)
    k, v = (_values((1, 60, heads, d), 21 + i, 0.7) for i in range(2))
    pk, pv = (_values((1, 90, heads, d), 23 + i, 0.7) for i in range(2))
    c.write(c.lists(table.cuda(), None, max_len=0), k.cuda(), v.cuda())
    c.write(c.lists(prefix.cuda(), None, max_len=0), pk.cuda(), pv.cuda())
    share = torch.full((batch,), -1, dtype=torch.int32)
    share[::50] = 0  # 14 columns: tiles of 16
    q = _values((batch, heads, d), 27, 0.3)
    own = c.lists(table.expand(batch, heads, 2).contiguous().cuda(), lens.cuda(), max_len=60)
    p = c.lists(prefix.cuda(), torch.full((1, heads), 90, dtype=torch.int32).cuda(), max_len=90)
    k, v, pk, pv = (_held(x[0], "int8") for x in (k, v, pk, pv))
    for _ in range(2):
        got = c.attn(own, q.cuda(), shared=p, share=share.cuda()).cpu().double()
        for b in list(range(0, 660, 50)) + [1, 333, 655, 656, 659]:
            there = torch.arange(60)[None] < lens[b][:, None]
            kb, vb = k, v
            if share[b] == 0:
                kb, vb = torch.cat((pk, k)), torch.cat((pv, v))
                there = torch.cat((torch.ones((heads, 90), dtype=torch.bool), there), 1)
            ref, _, tol, _ = _reference(q[b].double().view(heads, 1, d), kb, vb, there)
            assert float((got[b] - ref[:, 0]).abs().max()) <= tol, b


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,ptok,group,rows", ((128, 64, 16, 43), (64, 32, 7, 60), (128, 256, 2, 180),
                                              (64, 64, 13, 41), (128, 32, 1, 520)))
def test_prefixes_of_many_columns_that_may_be_long(kind, d, ptok, group, rows):
    # what the tables can hold, not the lengths, says that there is work for blocks of
    # 256 columns
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 60, (rows, 2), generator=g).tolist()
    s = Setup(kind, d, 2, lens, ptok=ptok, group=group, prefix_lens=[[4400, 97], [290, 0]], seed=d)
    l = s.lists[1]
    table = torch.full((2, 2, -(-60000 // ptok)), -1, dtype=torch.int32).cuda()
    table[:, :, :l.pages.shape[2]] = l.pages
    s.lists[1] = s.c.lists(table, l.length, max_len=60000)
    share = [(0, 0, 1, -1, 0)[i % 5] for i in range(rows)]
    s.check(share=share)
    s.check(share=[0] * (rows - 1) + [1])
    for i, (b, h, p) in enumerate(((0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1))):
        s.lists[1].pages[b, h, p] = (-1, s.c.cfg.num_pages, -7)[i]
    s.check(share=share, shared_first=[[1003, 96], [31, 5]],
            shared_dropped=[(0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1)])
