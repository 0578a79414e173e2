"""Norms with rotary positions against their formulas in 64 bits, and rows that go
straight into a paged cache against the same rows through two calls.

A result is held to half a step of bf16, 2^-8 of it, and to fp32's own errors (u =
2^-24): a mean of d values of at most x adds log2 d + 16 roundings and a square root and
a division few more, 32 u together; the norm's sums are of values less the mean, which is
off by 20 u max|x| itself; an angle is rounded at 1/2 turn, 2 pi 2^-26, a sine is off by
2^-22 and a turned value is a sum of two products: 2^-20 of the two.  So 2^-8 |y| and
2^-18 (the largest of the row, and the largest |x| by the norm's factor and weights).
"""
import math

import pytest
import torch

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.paged import PagedKV
from paper_2605_20600_amd.rotary import NormWeights, Rotary

pytestmark = pytest.mark.gpu


def _values(shape, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1] + (1,),
                                                                         generator=g))
    return x.to(torch.bfloat16)


def _omega(r, axes, base=10000.0):
    n = r // axes
    return [base ** (-2 * (j % (n // 2)) / n) for j in range(r // 2)]


def _want(x, positions, r, layout, axes, norm, weight, bias, eps=1e-6, scale=1.0, omega=None):
    """(result, bound) in 64 bits of x [rows][tokens][heads][d] (CPU)."""
    x = x.double()
    y, size = x, torch.zeros_like(x[..., :1])
    if norm:
        if norm == "layer":
            y = y - y.mean(-1, keepdim=True)
        f = 1 / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        y = y * f
        w = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight.double()
        size = x.abs().amax(-1, keepdim=True) * f * w.abs().amax(-1, keepdim=True)
        y = y * w
        if bias is not None:
            y = y + bias.double()
    y = y.clone()
    if r:
        c = positions.double().repeat_interleave(r // 2 // axes, -1)
        t = c * torch.tensor(omega or _omega(r, axes), dtype=torch.float64)
        # whole turns taken off where a cosine's own argument would be far
        t = torch.remainder(t, 2 * math.pi)[:, :, None]
        cos, sin = scale * torch.cos(t), scale * torch.sin(t)
        if layout == "half":
            a, b = y[..., :r // 2].clone(), y[..., r // 2:r].clone()
            y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = y[..., 0:r:2].clone(), y[..., 1:r:2].clone()
            y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, a * sin + b * cos
    bound = 2.0 ** -8 * y.abs() + 2.0 ** -18 * (1.5 * y.abs().amax(-1, keepdim=True) + size)
    return y, bound


def _check(got, want):
    y, bound = want
    off = (got.cpu().double() - y).abs()
    assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).max())


def _weights(kind, heads, d, seed, norm):
    if kind is None or norm is None:
        return None, None
    shape = (heads, d) if kind == "heads" else (d,)
    g = torch.Generator().manual_seed(seed)
    w = 1 + 0.3 * torch.randn(shape, generator=g)
    return w, (0.3 * torch.randn(shape, generator=g) if norm == "layer" else None)


def _gpu(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("d,r", ((64, 64), (64, 48), (64, 16), (128, 128), (128, 96), (128, 32),
                                 (128, 0)))
@pytest.mark.parametrize("layout", ("half", "pairs"))
@pytest.mark.parametrize("axes,norm,weights", ((1, None, None), (1, "rms", "heads"),
                                               (2, "layer", "one"), (2, "rms", None)))
def test_formula(d, r, layout, axes, norm, weights):
    rows, tokens, qh, kh = 3, 5, 11, 2
    q, k = _values((rows, tokens, qh, d), 1), _values((rows, tokens, kh, d), 2)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-5, 3000, (rows, tokens, axes), generator=g, dtype=torch.int32)
    rot = Rotary(d, r, layout=layout, axes=axes, norm=norm)
    qw, kw = _weights(weights, qh, d, 4, norm), _weights(weights, kh, d, 5, norm)
    got = rot(q.cuda(), k.cuda(), pos.cuda(),
              weights=NormWeights(*(_gpu(t) for t in (*qw, *kw))))
    _check(got[0], _want(q, pos, r, layout, axes, norm, *qw))
    _check(got[1], _want(k, pos, r, layout, axes, norm, *kw))


@pytest.mark.parametrize("rows,tokens,qh,kh", ((1, 1, 1, 0), (1, 1, 32, 32), (2, 700, 5, 1),
                                               (40, 3, 1, 20), (1, 4500, 20, 20)))
def test_sizes(rows, tokens, qh, kh):
    d = 64
    q, k = _values((rows, tokens, qh, d), 1), _values((rows, tokens, kh, d), 2) if kh else None
    pos = (torch.arange(tokens, dtype=torch.int32) + 7 * torch.arange(rows, dtype=torch.int32)[:, None])
    got = Rotary(d, norm="rms")(q.cuda(), _gpu(k), pos.cuda())
    _check(got[0], _want(q, pos[..., None], d, "half", 1, "rms", None, None))
    if kh:
        _check(got[1], _want(k, pos[..., None], d, "half", 1, "rms", None, None))
    else:
        assert got[1] is None


@pytest.mark.parametrize("layout", ("half", "pairs"))
def test_far_positions(layout):
    # angles whose whole turns are many: 64 bits leave 2^31 2^-53 of a turn
    d = 128
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 131072, -1, 0], dtype=torch.int32)
    x = _values((1, 6, 3, d), 8)
    got, _ = Rotary(d, layout=layout)(x.cuda(), None, pos.cuda()[None])
    # (the plain form's own angles are as large: exact fractions of a turn instead)
    from fractions import Fraction
    turns = B.headkv_rotary_plan(Rotary(d, layout=layout).cfg)
    rest = torch.tensor([[float((Fraction(t) * p) % 1) for t in turns] for p in pos.tolist()],
                        dtype=torch.float64)
    t = (rest * 2 * math.pi)[:, None]
    y = x[0].double()
    a, b = (y[..., :64], y[..., 64:]) if layout == "half" else (y[..., 0::2], y[..., 1::2])
    m, n = a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()
    want = torch.cat((m, n), -1) if layout == "half" else torch.stack((m, n), -1).flatten(-2)
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -18 * 1.5 * want.abs().amax(-1, keepdim=True)
    assert bool(((got[0].cpu().double() - want).abs() <= bound).all())


def test_scale_and_scalings():
    d, r = 128, 64
    x = _values((1, 9, 2, d), 1)
    pos = torch.arange(0, 90000, 10000, dtype=torch.int32)[None, :, None]
    for scaling in (("linear", 8.0), ("base", 8.0), ("bands", 8.0, 8192, 1.0, 4.0)):
        rot = Rotary(d, r, base=500000.0, scaling=scaling, scale=1.2079)
        omega = [2 * math.pi * t for t in B.headkv_rotary_plan(rot.cfg)]
        got, _ = rot(x.cuda(), None, pos.cuda())
        _check(got, _want(x, pos, r, "half", 1, None, None, None, scale=1.2079, omega=omega))
        # what does not turn is not scaled, and keeps its bits
        assert torch.equal(got[..., r:].cpu(), x[..., r:])


def test_rows_in_place_of_any_strides_behind_counts():
    rows, tokens, qh, kh, d = 4, 6, 6, 3, 128
    x = _values((rows, tokens, (qh + 2 * kh) * d + 8), 9).cuda()
    before = x.clone()
    q, k = (x[..., a * d:b * d].unflatten(2, (-1, d)) for a, b in ((0, qh), (qh, qh + kh)))
    pos = torch.arange(tokens, dtype=torch.int32).repeat(rows, 1)
    counts = torch.tensor([6, 0, 2, 9], dtype=torch.int32)
    rot = Rotary(d, norm="layer", layout="pairs")
    got = rot(q, k, pos.cuda(), counts=counts.cuda(), q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    want = before.cpu().clone().double()
    bound = torch.zeros_like(want)
    for a, b in ((0, qh), (qh, qh + kh)):
        y, e = _want(before[..., a * d:b * d].unflatten(2, (-1, d)).cpu(), pos[..., None], d,
                     "pairs", 1, "layer", None, None)
        for i, n in enumerate(counts.tolist()):
            want[i, :n, a * d:b * d] = y[i, :n].flatten(1)
            bound[i, :n, a * d:b * d] = e[i, :n].flatten(1)
    assert bool(((x.cpu().double() - want).abs() <= bound).all())
    # tokens and heads the other way round in memory
    t = _values((rows, qh, tokens, d), 10).cuda()
    got, _ = rot(t.transpose(1, 2), None, pos.cuda())
    _check(got, _want(t.transpose(1, 2).cpu(), pos[..., None], d, "pairs", 1, "layer", None, None))


def test_rows_that_are_no_numbers_stay_by_themselves():
    d = 64
    x = _values((1, 1, 40, d), 1)
    clean = x.clone()
    x[0, 0, 3, 60], x[0, 0, 17, 0], x[0, 0, 30, 5] = math.inf, math.nan, -math.inf
    pos = torch.full((1, 1), 5, dtype=torch.int32)
    for norm in (None, "rms", "layer"):
        rot = Rotary(d, 32, norm=norm)
        got, good = (rot(t.cuda(), None, pos.cuda())[0][0, 0].cpu() for t in (x, clean))
        others = [h for h in range(40) if h not in (3, 17, 30)]
        assert torch.equal(got[others], good[others])
        if norm is None:  # only what depends on it
            assert got[3, 60] == math.inf and torch.equal(got[3, :60], good[3, :60])
            assert not bool(got[17, [0, 16]].isfinite().any())
            assert torch.equal(got[17, 1:16], good[17, 1:16])
        elif norm == "layer":
            assert bool(got[[3, 17, 30]].isnan().all())
        else:
            assert bool(got[17].isnan().all())


def _cache(kind, d, heads, num_pages, **kw):
    c = PagedKV(kind, d, heads, num_pages, **kw)
    c.pool.fill_(255)
    return c


@pytest.mark.parametrize("kind", ("bf16", "int8", "fp4"))
@pytest.mark.parametrize("d,r,layout", ((64, 64, "half"), (64, 48, "half"), (64, 32, "pairs"),
                                        (128, 128, "half"), (128, 96, "half"), (128, 112, "half"),
                                        (128, 64, "pairs"), (128, 0, "half")))
@pytest.mark.parametrize("tokens,ragged", ((1, False), (4, True), (5, False), (37, True)))
def test_into_a_cache_as_in_two_calls(kind, d, r, layout, tokens, ragged):
    rows, kh, group, per = 5, 3, 2, 4
    qh = kh * group
    x = _values((rows, tokens, (qh + 2 * kh) * d), 3).cuda()
    x[0, 0, qh * d + 5] = math.inf   # a key row of no numbers, a value row, a row of zeros
    x[1, 0, (qh + kh) * d] = math.nan
    x[2, 0, qh * d:(qh + 1) * d] = 0
    q, k, v = (t.unflatten(2, (-1, d)) for t in x.split([qh * d, kh * d, kh * d], dim=2))
    g = torch.Generator().manual_seed(4)
    pages = torch.randperm(rows * kh * per, generator=g).to(torch.int32).view(rows, kh, per)
    pages[3, 1, 0], pages[4, 2, 1] = -1, 10 ** 6   # dropped ones
    pages = pages.cuda()
    length = torch.randint(0, 60, (rows, kh), generator=g, dtype=torch.int32)
    length[2] = torch.tensor([per * 32 - 1, per * 32, 0])  # the table's end
    length = length.cuda()
    pos = torch.randint(0, 5000, (rows, tokens), generator=g, dtype=torch.int32).cuda()
    counts = torch.tensor([tokens, 0, tokens, 1, tokens + 3], dtype=torch.int32).cuda() \
        if ragged else None
    rot = Rotary(d, r, layout=layout, norm="rms")
    weights = NormWeights(*(_gpu(t) for h in (qh, kh) for t in (_weights("heads", h, d, h, "rms"))))
    one, two = (_cache(kind, d, kh, rows * kh * per, page_tokens=32, group=group)
                for _ in range(2))
    lists = [c.lists(pages, length, max_len=60, extra=2) for c in (one, two)]
    got = one.write_rotary(lists[0], rot, q, k, v, pos, weights=weights, counts=counts)
    want_q, want_k = rot(q, k, pos, weights=weights, counts=counts)
    two.write(lists[1], want_k, v.contiguous(), counts=counts)
    assert torch.equal(got.view(torch.int16), want_q.view(torch.int16))
    assert torch.equal(one.pool, two.pool)
    assert bool((one.pool != 255).any())
    # without queries
    one.pool.fill_(255)
    assert one.write_rotary(lists[0], rot, None, k, v, pos, weights=weights, counts=counts) is None
    assert torch.equal(one.pool, two.pool)


def test_other_streams_and_replays():
    d, rows = 128, 8
    rot = Rotary(d, norm="rms")
    x = _values((rows, 1, 96, d), 1).cuda()
    q, k, v = x.split(32, dim=2)
    cache = _cache("int8", d, 32, rows * 32)
    pages = torch.arange(rows * 32, dtype=torch.int32).view(rows, 32, 1).cuda()
    length = torch.zeros((rows, 32), dtype=torch.int32, device="cuda")
    lists = cache.lists(pages, length, max_len=64)
    pos = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.write_rotary(lists, rot, q, k, v, pos, q_out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.write_rotary(lists, rot, q, k, v, pos, q_out=out)
        length += 1
        pos += 3
    for step in range(4):
        torch.cuda.synchronize()
        x.copy_(_values(x.shape, 20 + step))
        want = rot(q, k, torch.full_like(pos, 3 * step))
        graph.replay()
        assert torch.equal(out, want[0])
        assert int(length[0, 0]) == step + 1
        plain = _cache("int8", d, 32, rows * 32)
        plain.write(plain.lists(pages, torch.full_like(length, step), max_len=64), want[1], v.contiguous())
        a, b = (c.read(c.lists(pages, length, max_len=64), 1, begin=-1) for c in (cache, plain))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rows_far_apart():
    # offsets past 2^31 elements, in and out
    d = 64
    buf = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 1, 3, d), (1 << 31, d * 3, d, 1))
    x.copy_(_values((2, 1, 3, d), 1))
    want = x.clone()
    pos = torch.tensor([[3], [4]], dtype=torch.int32)
    Rotary(d)(x, None, pos.cuda(), q_out=x)
    _check(x, _want(want.cpu(), pos[..., None], d, "half", 1, None, None, None))


def test_refusals():
    rot = Rotary(64, norm="rms")
    x = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    ok = dict(q=x, k=x, positions=pos)
    bad = [dict(q=x.float()), dict(q=x.cpu()), dict(k=x[:, :2]), dict(q=x[..., :32]),
           dict(positions=pos.long()), dict(positions=pos[:1]), dict(positions=None),
           dict(positions=pos.cpu()), dict(counts=pos[:1, 0]), dict(q=None, k=None),
           dict(q_out=x[:1]), dict(q_out=x.cpu()), dict(q=x.transpose(2, 3)),
           dict(weights=NormWeights(torch.ones(32, device="cuda"))),
           dict(weights=NormWeights(k_bias=torch.ones((5, 64), device="cuda")))]
    for w in ((torch.ones(64, device="cuda").double(),), (torch.ones(64),),
              (torch.ones(64, device="cuda"), torch.ones((4, 64), device="cuda")),
              (torch.ones((64, 4), device="cuda").t(),), (torch.ones((1, 4, 64), device="cuda"),)):
        with pytest.raises(ValueError):
            NormWeights(*w)
    for kw in bad:
        with pytest.raises(ValueError):
            rot(**{**ok, **kw})
    with pytest.raises(B.HeadKVError):  # rows that would be written twice
        rot(x, None, pos, q_out=x[:1].expand(2, -1, -1, -1))
    with pytest.raises(ValueError):
        Rotary(64, layout="other")
    with pytest.raises(ValueError):
        Rotary(64, scaling=("linear",))
    with pytest.raises(B.HeadKVError):
        Rotary(96)
    c = PagedKV("int8", 64, 4, 8, group=1)
    lists = c.lists(torch.zeros((2, 4, 1), dtype=torch.int32, device="cuda"), None, max_len=0)
    for kw in (dict(q=x[:, :, :2]), dict(k=x[:, :, :2]), dict(v=x[:1]), dict(v=x.float()),
               dict(counts=pos), dict(positions=None)):
        with pytest.raises(ValueError):
            c.write_rotary(**{**dict(lists=lists, rotary=rot, q=x, k=x, v=x, positions=pos), **kw})
    # nothing to write
    assert c.write_rotary(lists, rot, x[:, :0], x[:, :0], x[:, :0], pos[:, :0]).shape[1] == 0


def test_other_devices(monkeypatch):
    # nothing is launched unless every tensor and the current device are one (another device
    # is stood in for: the check runs before anything is launched)
    from paper_2605_20600_amd import paged
    from paper_2605_20600_amd.drafts import verify_drafts
    from paper_2605_20600_amd.page_tables import PageTables
    rot = Rotary(64)
    x = torch.ones((1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    cache = _cache("bf16", 64, 2, 6, page_tokens=32)
    lists = cache.lists(torch.arange(6, dtype=torch.int32, device="cuda").view(1, 2, 3), None, 0)
    tables = PageTables(2, 3, 6, 1)
    logits = torch.zeros((1, 2, 9), device="cuda")
    state = [t.clone() for t in (x, cache.pool, tables.buffer)]
    monkeypatch.setattr(paged, "_current_device", lambda: cache.index + 1)
    for f in (lambda: rot(x, None, pos, q_out=x), lambda: tables.extend(3),
              lambda: cache.write_rotary(lists, rot, x, x, x, pos),
              lambda: cache.attn_tokens(lists, x),
              lambda: verify_drafts(logits, pos[:, :1], logits[:, :, 0].contiguous())):
        with pytest.raises(ValueError, match="current device"):
            f()
    torch.cuda.synchronize()
    for a, b in zip(state, (x, cache.pool, tables.buffer)):
        assert torch.equal(a, b)
    monkeypatch.undo()
    other = cache.lists(lists.pages, None, 0)
    cache.index += 1
    for f in (lambda: cache.write_rotary(other, rot, x, x, x, pos),
              lambda: cache.attn_tokens(other, x)):
        with pytest.raises(ValueError):
            f()
