"""Verification of drafted tokens against the same steps one after the other in 64 bits.

Tokens and counts have to be equal: a decision is turned by sums of 64 bits only where a
uniform lies within some 2^-45 of a border.  A log probability is held to half a step of
fp32, 2^-24 of it, and 2^-40 for the 64-bit sums.
"""
import math

import pytest
import torch

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.drafts import verify_drafts

pytestmark = pytest.mark.gpu
TOP = 1 - 2.0 ** -24


def _oracle(logits, tokens, uniforms, draft=None, counts=None, t=1.0):
    """Row by row, draft by draft (CPU tensors)."""
    rows, drafts = tokens.shape
    vocab = logits.shape[2]
    kept = torch.full((rows, drafts + 1), -1, dtype=torch.int32)
    logprob = torch.zeros((rows, drafts + 1), dtype=torch.float64)
    count = torch.zeros(rows, dtype=torch.int32)
    for r in range(rows):
        given = drafts if counts is None else min(int(counts[r]), drafts)
        if given < 0:
            continue
        for i in range(drafts + 1):
            x = logits[r, i].double()
            token = int(tokens[r, i]) if i < given else -1
            is_draft = 0 <= token < vocab
            if bool(x.isnan().any()) or float(x.max()) in (math.inf, -math.inf):
                break
            q = torch.zeros(vocab, dtype=torch.float64)
            if t == 0:
                p = torch.zeros(vocab, dtype=torch.float64)
                p[int((x == x.max()).nonzero()[0])] = 1
            else:
                p = torch.softmax((x - x.max()) / t, 0)
                if is_draft and draft is None:
                    q[token] = 1
                elif is_draft:
                    y = draft[r, i].double()
                    if bool(y.isnan().any()) or float(y.max()) == math.inf:
                        break
                    if float(y.max()) > -math.inf:
                        q = torch.softmax((y - y.max()) / t, 0)
            u = float(uniforms[r, i])
            if is_draft and u < 1 and max(u, 0.0) * float(q[token]) < float(p[token]):
                kept[r, i] = token
                logprob[r, i] = math.log(float(p[token]))
                count[r] += 1
                continue
            rest = (p - q).clamp(min=0)
            if float(rest.sum()) < 2.0 ** -40:
                rest = p
            up = rest.cumsum(0)
            u = float(uniforms[r, drafts])
            u = max(u, 0.0) if u < 1 else TOP
            token = int(torch.searchsorted(up, u * up[-1:], right=True)[0])
            if token >= vocab or float(rest[token]) == 0:
                token = int(rest.nonzero()[-1])
            kept[r, i] = token
            logprob[r, i] = math.log(float(p[token]))
            count[r] += 1
            break
    return kept, count, logprob


def _check(logits, tokens, uniforms, draft=None, counts=None, t=1.0):
    want, count, logprob = _oracle(logits.cpu(), tokens, uniforms, None if draft is None
                                   else draft.cpu(), counts, t)
    got = verify_drafts(logits, tokens.cuda(), uniforms.cuda(), draft_logits=draft,
                        counts=None if counts is None else counts.cuda(), temperature=t)
    assert torch.equal(got["tokens"].cpu(), want)
    assert torch.equal(got["count"].cpu(), count)
    off = (got["logprob"].cpu().double() - logprob).abs()
    assert bool((off <= 2.0 ** -24 * logprob.abs() + 2.0 ** -40).all()), float(off.max())
    return want, count


def _inputs(rows, drafts, vocab, dtype, seed, model=True, near=0.5, spread=2.5, masked=0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((rows, drafts + 1, vocab), generator=g)
    x[..., :masked] = -math.inf
    y = x[:, :drafts] + near * torch.randn((rows, drafts, vocab), generator=g)
    pick = y if model else 3 * x[:, :drafts]
    tokens = torch.zeros((rows, drafts), dtype=torch.int32)
    if drafts:
        noise = torch.empty_like(pick).exponential_(generator=g).log()
        tokens = (pick - noise).argmax(2).to(torch.int32)
    return (x.to(dtype), tokens, torch.rand((rows, drafts + 1), generator=g),
            y.to(dtype) if model else None)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("rows,drafts,vocab", (
    (1, 0, 1), (3, 1, 1), (5, 2, 2), (4, 3, 7), (9, 4, 1000), (2, 1, 2041), (2, 2, 2049),
    (3, 5, 8185), (2, 3, 16389), (1, 63, 300), (30, 4, 8192), (2, 1, 65536), (300, 1, 40)))
@pytest.mark.parametrize("model", (True, False))
def test_sizes(dtype, rows, drafts, vocab, model):
    x, tokens, u, y = _inputs(rows, drafts, vocab, dtype, rows + vocab, model)
    _check(x.cuda(), tokens, u, None if y is None else y.cuda())


def test_long_rows_of_many():
    # where a block takes 8192 logits
    x, tokens, u, y = _inputs(40, 4, 30001, torch.bfloat16, 5)
    _check(x.cuda(), tokens, u, y.cuda(), t=0.8)
    x, tokens, u, _ = _inputs(24, 4, 60000, torch.float32, 6, model=False)
    _check(x.cuda(), tokens, u, t=0.8)


@pytest.mark.parametrize("t", (0.0, 0.01, 0.7, 3.0, 1e5))
@pytest.mark.parametrize("model", (True, False))
def test_temperatures_and_masks(t, model):
    x, tokens, u, y = _inputs(12, 4, 5000, torch.bfloat16, 8, model, masked=4000)
    kept, count = _check(x.cuda(), tokens, u, None if y is None else y.cuda(), t=t)
    assert bool((kept[kept >= 0] >= 4000).all())
    if t == 0:  # greedy drafts are kept
        best = x.float().argmax(2).to(torch.int32)
        kept, count = _check(x.cuda(), best[:, :4].contiguous(), u, t=0)
        assert torch.equal(kept, best) and int(count.min()) == 5


def test_counts_and_tokens_that_are_none():
    x, tokens, u, y = _inputs(8, 4, 600, torch.float32, 9, near=0.05)
    tokens[2, 1], tokens[3, 0], tokens[4, 3], tokens[5, 2] = -1, 600, 2 ** 31 - 1, -2 ** 31
    counts = torch.tensor([0, -1, 4, 9, 2, 4, -7, 3], dtype=torch.int32)
    for t in (1.0, 0.0):
        for draft in (None, y.cuda()):
            kept, count = _check(x.cuda(), tokens, u, draft, counts, t)
            assert count[1] == 0 and count[6] == 0 and count[0] == 1 and count[3] == 1


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_strides_and_alignments(dtype):
    x, tokens, u, y = _inputs(3, 4, 4100, dtype, 10)
    big = torch.full((3, 5, 4113), math.nan, dtype=dtype, device="cuda")
    for start in (0, 1, 3, 5, 8):
        a = big[..., start:start + 4100]
        a.copy_(x)
        # drafts' rows before those of other positions, read backwards in memory
        b = torch.full((4, 3, 4107), math.nan, dtype=dtype, device="cuda")[..., 7:]
        b.copy_(y.transpose(0, 1))
        _check(a, tokens, u, b.transpose(0, 1))
        big.fill_(math.nan)
    # one row of logits for all
    same = x[:1].cuda().expand(3, -1, -1)
    _check(same, tokens, u, y.cuda())


def test_rows_that_are_no_numbers():
    x, tokens, u, y = _inputs(12, 3, 900, torch.float32, 11, near=0.02)
    u[:, :3] = 0  # every draft with p > 0 is kept
    x[0, 0, 5], x[1, 1, 899], x[2, 3, 0], x[3, 2] = math.nan, math.inf, math.nan, -math.inf
    y[4, 0, 7], y[5, 2, 8] = math.nan, math.inf
    y[6, 1] = -math.inf              # stands for q = 0
    x[7, 2, int(tokens[7, 2])] = -math.inf  # p = 0: not kept, and not drawn
    x[8, 3] = -math.inf
    tokens[9, 1] = -1                # nothing behind it is looked at
    x[9, 2:] = math.nan
    x[10, :, 3] = -math.inf
    counts = torch.full((12,), 3, dtype=torch.int32)
    for draft in (y.cuda(), None):
        kept, count = _check(x.cuda(), tokens, u, draft, counts)
        assert count.tolist()[:4] == [0, 1, 3, 2] and int(count[8]) == 3
    _check(x.cuda(), tokens, u, None, counts, t=0.0)


def test_distributions_that_are_the_same():
    # q = p keeps everything, the largest uniform included
    x, tokens, u, _ = _inputs(6, 4, 3000, torch.bfloat16, 12)
    u[:, :4] = TOP
    kept, count = _check(x.cuda(), tokens, u, x[:, :4].contiguous().cuda())
    assert int(count.min()) == 5
    # a draft that neither gives any probability: what follows is drawn from p
    x[:, 0, 17] = -math.inf
    tokens[:, 0] = 17
    kept, count = _check(x.cuda(), tokens, u, x[:, :4].contiguous().cuda())
    assert int(count.max()) == 1


def test_uniforms_at_the_borders():
    x, tokens, u, y = _inputs(8, 2, 50, torch.float32, 13)
    for first, last in ((0.0, 0.0), (TOP, TOP), (0.0, TOP), (TOP, 0.0), (1.0, 1.0),
                        (math.nan, math.nan), (-1.0, -0.5), (2.0, 3.0)):
        u[:, :2], u[:, 2] = first, last
        for draft in (y.cuda(), None):
            kept, count = _check(x.cuda(), tokens, u, draft)
            if not first < 1:
                assert int(count.max()) == 1
    # exact halves: up to u = 1/2 the first, from there on the second
    x = torch.zeros((3, 1, 2))
    u = torch.tensor([[0.5 - 2.0 ** -25], [0.5], [0.5 + 2.0 ** -24]])
    kept, _ = _check(x.cuda(), torch.zeros((3, 0), dtype=torch.int32), u)
    assert kept[:, 0].tolist() == [0, 1, 1]


@pytest.mark.parametrize("size", (1e4, 1e30, 3e38))
def test_large_logits(size):
    g = torch.Generator().manual_seed(14)
    x = size * (torch.rand((4, 3, 700), generator=g) * 2 - 1)
    x[:, :, 5:9] = x.amax(2, keepdim=True)  # equal largest ones
    tokens = torch.full((4, 2), 6, dtype=torch.int32)
    u = torch.rand((4, 3), generator=g)
    for t in (1.0, 0.0, 1e30):
        _check(x.cuda(), tokens, u, t=t)
        _check(x.cuda(), tokens, u, x[:, :2].contiguous().flip(2).cuda(), t=t)


def test_what_comes_out_is_the_targets():
    # 200000 rows of one target and one draft: the first token's share is p (5 deviations of
    # a share of n, sqrt(p (1 - p) / n), for 12 tokens; a sixth of them would be seen)
    n, vocab = 200000, 12
    g = torch.Generator(device="cuda").manual_seed(15)
    x = torch.randn((1, 2, vocab), generator=g, device="cuda")
    y = torch.randn((1, 1, vocab), generator=g, device="cuda")
    tokens = torch.multinomial(torch.softmax(y[0, 0], 0), n, replacement=True, generator=g)
    u = torch.rand((n, 2), generator=g, device="cuda")
    got = verify_drafts(x.expand(n, -1, -1), tokens.to(torch.int32)[:, None].contiguous(), u,
                        draft_logits=y.expand(n, -1, -1))
    p = torch.softmax(x[0, 0].double(), 0)
    share = torch.bincount(got["tokens"][:, 0].long(), minlength=vocab).double() / n
    assert bool(((share - p).abs() < 5 * (p * (1 - p) / n).sqrt()).all())
    # and the second one's, where there is one
    second = got["tokens"][got["count"] == 2, 1].long()
    p = torch.softmax(x[0, 1].double(), 0)
    share = torch.bincount(second, minlength=vocab).double() / len(second)
    assert bool(((share - p).abs() < 5 * (p * (1 - p) / len(second)).sqrt()).all())


def test_more_rows_than_a_launch():
    # 2^24 / (3 * segments) rows a launch, and more than there are counters
    n = (1 << 16) + 5
    g = torch.Generator().manual_seed(16)
    x = torch.randn((7, 2, 30), generator=g)
    tokens = torch.randint(0, 30, (n, 1), generator=g, dtype=torch.int32)
    u = torch.rand((n, 2), generator=g)
    pick = torch.arange(n) % 7
    got = verify_drafts(x[pick].cuda(), tokens.cuda(), u.cuda())
    some = torch.cat((torch.arange(50), torch.arange(n - 50, n)))
    kept, count, _ = _oracle(x[pick[some]], tokens[some], u[some])
    assert torch.equal(got["tokens"].cpu()[some], kept)
    assert torch.equal(got["count"].cpu()[some], count)


def test_replays_and_streams():
    x, tokens, u, y = (t.cuda() for t in _inputs(16, 4, 20000, torch.bfloat16, 17))
    eager = verify_drafts(x, tokens, u, draft_logits=y)
    eager = {k: v.clone() for k, v in eager.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = verify_drafts(x, tokens, u, draft_logits=y)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs, each its own workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, verify_drafts(x, tokens, u, draft_logits=y)))
    for k in eager:
        assert torch.equal(eager[k], other[k])
    for i in range(4):
        u.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(i)))
        want = verify_drafts(x, tokens, u, draft_logits=y)
        for graph, got in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph, got in graphs:
            for k in want:
                assert torch.equal(want[k], got[k])


def test_refusals():
    x, tokens, u, y = (t.cuda() for t in _inputs(2, 3, 50, torch.bfloat16, 18))
    ok = dict(logits=x, tokens=tokens, uniforms=u, draft_logits=y)
    bad = [dict(logits=x.half()), dict(logits=x.cpu()), dict(logits=x[0]), dict(logits=x[:, :0]),
           dict(logits=x.transpose(1, 2)), dict(tokens=tokens.long()), dict(tokens=tokens[:, :2]),
           dict(uniforms=u[:, :3]), dict(uniforms=u.double()), dict(uniforms=u.cpu()),
           dict(draft_logits=y.float()), dict(draft_logits=y[:, :2]), dict(draft_logits=y.cpu()),
           dict(counts=tokens), dict(counts=tokens[:, 0].cpu())]
    for kw in bad:
        with pytest.raises(ValueError):
            verify_drafts(**{**ok, **kw})
    with pytest.raises(B.HeadKVError):
        verify_drafts(**ok, temperature=-1.0)
    got = verify_drafts(x[:0], tokens[:0], u[:0])
    assert got["tokens"].shape == (0, 4) and got["count"].shape == (0,)
