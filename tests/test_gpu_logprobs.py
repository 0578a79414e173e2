"""headkv_token_logprobs against a 64-bit implementation.

Bounds: a lane sums at most vocab / 64 + 64 terms one after the other and the
rest is a tree, so log S is off by at most (vocab / 64 + 80) 2^-23 + 2^-20 (the
exponentials), and y - m by 2 roundings of it: for log p
(vocab / 64 + 80) 2^-23 + 2^-20 + 2^-22 |log p|.  The entropy is log S minus a
mean of (y - m) under the weights, off by as much relatively as they are: the
same with (1 + H + largest |y - m| that has weight) in front."""
import math

import pytest
import torch

from paper_2605_20600_amd.paged import token_logprobs

pytestmark = pytest.mark.gpu


def _check(x, tokens, top, temperature=1.0, x_dev=None, got=None):
    if got is None:
        got = token_logprobs(x.cuda() if x_dev is None else x_dev, tokens.cuda(), top=top,
                             temperature=temperature)
    got = {k: v.cpu() for k, v in got.items()}
    rows, vocab = x.shape
    raw = x.double()
    bad = (raw.isnan() | (raw == math.inf)).any(1)
    ok = ~bad
    for key in got:
        if key in ("rank", "top_index"):
            assert bool((got[key][bad] == -1).all())
        else:
            assert bool(got[key][bad].isnan().all())
    lp = torch.log_softmax(raw / temperature, 1)
    empty = (raw == -math.inf).all(1)
    lp[empty] = -math.inf
    base = (vocab / 64 + 80) * 2.0 ** -23 + 2.0 ** -20

    def near(a, b):
        a, b = a.double(), b
        inf = b == -math.inf
        assert torch.equal(a == -math.inf, inf)
        err = (a - b)[~inf].abs()
        assert bool((err <= base + 2.0 ** -22 * b[~inf].abs()).all()), float(err.max())

    has = (tokens >= 0) & (tokens < vocab)
    at = tokens.long().clamp(0, vocab - 1)[:, None]
    want = torch.where(has, lp.gather(1, at)[:, 0], -math.inf)
    near(got["logprob"][ok], want[ok])
    rank = torch.where(has, (raw > raw.gather(1, at)).sum(1), -1).to(torch.int32)
    assert torch.equal(got["rank"][ok], rank[ok])
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    spread = torch.where(p > 2.0 ** -40, lp.amax(1, keepdim=True) - lp, 0).amax(1)
    err = (got["entropy"].double() - h)[ok].abs()
    assert bool((err <= base * (1 + h + spread)[ok]).all()), float(err.max())
    if top:
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got["top_index"][ok], order[ok].to(torch.int32))
        near(got["top_logprob"][ok], lp.gather(1, order)[ok])
    else:
        assert "top_index" not in got


def _logits(rows, vocab, dtype, seed, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (scale * torch.randn((rows, vocab), generator=g)).to(dtype)
    return x, torch.randint(0, vocab, (rows,), generator=g).to(torch.int32)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("rows,vocab,top", (
    (1, 1, 1), (1, 2, 0), (3, 7, 5), (5, 33, 32), (2, 1000, 20), (7, 4095, 5), (4, 4096, 32),
    (3, 4097, 7), (300, 1500, 3), (2, 16384, 0), (9, 16385, 32), (1, 65536, 32), (2, 131071, 11)))
def test_scores(dtype, rows, vocab, top):
    x, t = _logits(rows, vocab, dtype, rows + vocab)
    _check(x, t, top)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("temperature", (0.1, 0.7, 5.0))
def test_temperature(dtype, temperature):
    x, t = _logits(6, 5000, dtype, 1)
    _check(x, t, 8, temperature)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("vocab", (50, 6000, 40000))
def test_masked_infinite_and_nan_rows(dtype, vocab):
    x, t = _logits(12, vocab, dtype, 2)
    x[0] = -math.inf                      # nothing left
    x[1, 1:] = -math.inf                  # one token left
    x[2, :vocab - 3] = -math.inf          # fewer left than alternatives asked
    x[3] = torch.finfo(dtype).min         # the type's lowest value everywhere
    x[4, :vocab // 2] = torch.finfo(dtype).min
    x[5, vocab // 3] = math.nan
    x[6, vocab - 1] = math.inf
    x[7, 0] = -math.nan
    x[8, 7] = 0.0
    x[8, 8] = -0.0                        # equal to the one before
    x[8, :7] = -1.0
    x[9] = 0.25                           # all equal
    x[10, 13] = torch.finfo(dtype).max    # the rest has no weight
    t[0], t[1], t[2], t[10] = 3, 2, vocab - 2, 13
    _check(x, t, 32)
    _check(x, t, 0)
    t[4], t[8], t[9], t[11] = -1, vocab, 2 ** 31 - 1, -2 ** 31
    _check(x, t, 1)


@pytest.mark.parametrize("order", ("up", "down", "ends", "blocks"))
def test_orders_that_a_selection_may_mind(order):
    vocab = 20000
    x = torch.linspace(-5, 5, vocab).repeat(2, 1)
    if order == "down":
        x = x.flip(1).contiguous()
    if order == "ends":
        x[:, 1000:-1000] = -20
    if order == "blocks":  # the largest all next to each other, and in one stride
        x = -x.abs()
        x[0, 8192:8192 + 40] = torch.arange(40.0)
        x[1, ::512] = torch.arange(40.0)
    _check(x, torch.tensor([5, vocab - 1], dtype=torch.int32), 32)
    _check(x.to(torch.bfloat16), torch.tensor([5, vocab - 1], dtype=torch.int32), 32)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_rows_of_any_stride_and_alignment(dtype):
    x, t = _logits(5, 3001, dtype, 3)
    for lead in (0, 1, 3):
        wide = torch.full((5, 3500), math.nan, dtype=dtype, device="cuda")
        view = wide[:, lead:lead + 3001]
        view.copy_(x)
        _check(x, t, 9, x_dev=view)


def test_row_offsets_past_32_bits():
    rows, vocab = 40, 1000
    x, t = _logits(rows, vocab, torch.bfloat16, 4)
    wide = torch.empty((rows, 120_000_000), dtype=torch.bfloat16, device="cuda")
    view = wide[:, :vocab]
    view.copy_(x)
    assert wide.numel() > 1 << 32
    _check(x, t, 3, x_dev=view)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_a_very_long_row(dtype):
    x, t = _logits(2, (1 << 21) + 5, dtype, 8)
    x[1, :1 << 20] = -math.inf
    t[1] = (1 << 21) + 4
    _check(x, t, 32)


def test_many_rows_and_repeats_are_the_same():
    x, t = _logits(5000, 2000, torch.bfloat16, 5)
    _check(x, t, 2)
    xd, td = x.cuda(), t.cuda()
    first = token_logprobs(xd, td, top=2)
    for _ in range(3):
        again = token_logprobs(xd, td, top=2)
        for k in first:
            assert torch.equal(first[k], again[k])


def test_calls_of_any_sizes_share_the_workspace():
    # what a call leaves behind its counters may not be taken for another's counters
    for rows, vocab, top in ((256, 65536, 32), (1500, 17000, 1), (3, 300000, 32), (6000, 16500, 0),
                             (40, 70000, 20), (256, 65536, 32)):
        x, t = _logits(rows, vocab, torch.bfloat16, rows)
        _check(x, t, top)


def test_more_rows_than_counters():
    g = torch.Generator().manual_seed(9)
    rows, vocab = 65536 + 300, 16500
    one = (3 * torch.randn((1, vocab), generator=g)).to(torch.bfloat16)
    x = one.expand(rows, vocab).contiguous()
    x[:, 0] = torch.linspace(0, 20, rows).to(torch.bfloat16)
    t = torch.randint(0, vocab, (rows,), generator=g).to(torch.int32)
    got = token_logprobs(x.cuda(), t.cuda(), top=2)
    some = torch.tensor([0, 1, 65535, 65536, 65537, rows - 1])
    _check(x[some], t[some], 2, got={k: v[some.cuda()] for k, v in got.items()})


def test_on_another_stream_and_in_a_graph():
    x, t = _logits(4, 70000, torch.bfloat16, 6)
    xd, td = x.cuda(), t.cuda()
    want = token_logprobs(xd, td, top=4)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = token_logprobs(xd, td, top=4)
    st.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k])
    with torch.cuda.stream(st):  # the capture's stream has its workspace
        token_logprobs(xd, td, top=4)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        res = token_logprobs(xd, td, top=4)
    for i in range(4):
        xd.copy_((x.float() * (1 + i)).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        now = {k: v.clone() for k, v in res.items()}
        eager = token_logprobs(xd, td, top=4)
        for k in now:
            assert torch.equal(now[k], eager[k]), (i, k)


def test_refusals():
    x = torch.zeros((2, 10), device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((x.double(), t), (x[:, ::2], t), (x, t.long()), (x[0], t)):
        with pytest.raises(ValueError):
            token_logprobs(*args)


def test_refuses_host_memory():
    x = torch.zeros((2, 10), device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((x.cpu(), t), (x, t.cpu())):
        with pytest.raises(ValueError):
            token_logprobs(*args)


def test_first_use_in_a_graph():
    # the workspace that a capture makes belongs to the graph alone
    x, t = _logits(5, 70000, torch.float32, 8)
    xd, td = x.cuda(), t.cuda()
    want = token_logprobs(xd, td, top=7)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        res = token_logprobs(xd, td, top=7)
    with torch.cuda.stream(st):  # before any replay
        eager = token_logprobs(xd, td, top=7)
    st.synchronize()
    for k in want:
        assert torch.equal(eager[k], want[k]), k
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(res[k], want[k]), k
        token_logprobs(xd, td, top=7)
