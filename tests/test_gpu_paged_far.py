"""Paged attention of scores from 2^24 (log2 units) on, where a running maximum and the
scores less it are rounded alike, and of lists that reach them on the way.

Keys and queries have one component that is not zero, powers of two, so that scores are
exact products.  Where the largest is large, the tokens that share it have all the
weight: the output is the mean of their values, off by (n + 8) 2^-23 of the largest value,
and the log of the sum is the score (rounded: the scale to log2 units, the product, back
to nats: 2^-22 of it) plus the log of their number.  Tokens with other scores s and weight (s - max >= -60, else under 2^-86) are off
by 2^-20, the exponential, and 4 |s - max| 2^-23, the scale, the product and two
differences, relatively; twice that in the mean."""
import math

import pytest
import torch

from test_gpu_paged import TYPES, U, _cache, _held, _values

pytestmark = pytest.mark.gpu


def _far(kind, d, scores, group=1, share=None, prefix=None, ptok=64, seed=0):
    """scores [rows][tokens] and prefix [prefixes][tokens]: of query times key, powers of two
    of either sign, q being 2^20 of them at most."""
    sets = [scores] + ([] if prefix is None else [prefix])
    per = [-(-x.shape[1] // ptok) for x in sets]
    heads = 2
    c = _cache(kind, d, heads, sum(len(x) * heads * p for x, p in zip(sets, per)), page_tokens=ptok,
               group=group)
    tables = torch.arange(c.cfg.num_pages, dtype=torch.int32).cuda()
    at, lists, held = 0, [], []
    dims = (5, d - 1)  # of each head
    for i, (x, p) in enumerate(zip(sets, per)):
        n = len(x) * heads * p
        table = tables[at:at + n].view(len(x), heads, p).contiguous()
        at += n
        k = torch.zeros((*x.shape, heads, d), dtype=torch.bfloat16)
        for h in range(heads):
            k[:, :, h, dims[h]] = (x / 2.0 ** 20).to(torch.bfloat16)
        v = _values(k.shape, seed + i, 0.7)
        assert torch.equal(k.sum(-1)[:, :, 0].double() * 2.0 ** 20, x)
        c.write(c.lists(table, None, max_len=0), k.cuda(), v.cuda())
        length = torch.full((len(x), heads), x.shape[1], dtype=torch.int32).cuda()
        lists.append(c.lists(table, length, max_len=x.shape[1]))
        held.append((_held(k, kind), _held(v, kind)))
    rows = len(scores)
    q = torch.zeros((rows, heads, group, d), dtype=torch.bfloat16)
    for h in range(heads):
        q[:, h, :, dims[h]] = 2.0 ** 20
    q = q.view(rows, heads * group, d)
    lse = torch.empty((rows, heads * group), device="cuda")
    kw = {} if prefix is None else dict(shared=lists[1], share=torch.tensor(
        share, dtype=torch.int32).cuda())
    out = c.attn(lists[0], q.cuda(), lse=lse, **kw).cpu().double()
    lse = lse.cpu().double()
    for b in range(rows):
        for h in range(heads):
            k, v = (x[b, :, h] for x in held[0])
            if prefix is not None and share[b] >= 0:
                k, v = (torch.cat((y[share[b], :, h], x)) for x, y in zip((k, v), held[1]))
            s = k[:, dims[h]] * 2.0 ** 20 / math.sqrt(d)
            less = s - s.max()
            want = torch.softmax(less, 0) @ v
            want_lse = float(s.max() + torch.logsumexp(less, 0))
            weighed = less >= -60
            e = 0.0
            if bool((less[weighed] < 0).any()):
                e = 2.0 ** -20 + 4 * float(less[weighed].abs().max()) * U
            got = out[b].view(heads, group, d)[h]
            tol = (2 * e + (len(k) + 8) * U) * float(v[weighed].abs().max())
            assert float((got - want).abs().max()) <= tol, (b, h)
            err = (lse[b].view(heads, group)[h] - want_lse).abs().max()
            assert float(err) <= 2.0 ** -22 * abs(want_lse) + e + (len(k) + 8) * U, (b, h)


def _scores(exponent, sign, tokens, seed):
    """Fewest and most likely ones a factor of four apart."""
    g = torch.Generator().manual_seed(seed)
    c = 2.0 ** -torch.randint(0, 3, (3, tokens), generator=g).double()
    return sign * c * 2.0 ** exponent


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("sign", (-1, 1))
def test_large_scores_of_own_lists(kind, d, sign):
    for exponent in (16, 25, 27, 28, 31, 34, 36, 40, 60, 100):
        _far(kind, d, _scores(exponent, sign, 300, exponent), seed=exponent)
    _far(kind, d, _scores(35, sign, 3000, 1), group=3)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rising", (True, False))
def test_scores_that_become_large(kind, rising):
    # from 1 to 2^60 and back, of both signs, the largest in the last or the first step
    tokens = 1500
    e = torch.arange(tokens).mul(60).div(tokens - 1, rounding_mode="floor").double()
    x = torch.stack((2.0 ** e, -2.0 ** (60 - e), 2.0 ** (e / 2).floor()))
    _far(kind, 128, x if rising else x.flip(1), seed=3)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,group", ((3, 1), (20, 2)))
def test_large_scores_beside_prefixes(kind, rows, group):
    # the prefix's scores as large as the list's, larger, smaller and ordinary
    own = torch.cat([_scores(e, s, 200, e) for e, s in ((30, 1), (45, -1), (4, 1), (60, 1), (26, -1),
                                                        (33, 1), (2, -1))])[:rows]
    prefix = torch.cat([_scores(e, s, 700, e)[:1] for e, s in ((30, 1), (34, -1), (62, 1), (3, 1))])
    _far(kind, 128, own, group=group, prefix=prefix, seed=5,
         share=[(0, 1, 2, 3, -1)[i % 5] for i in range(rows)])


@pytest.mark.parametrize("kind", TYPES)
def test_large_scores_of_blocks_of_many_columns(kind):
    # 16 heads a row, so that the prefix has hundreds of columns, and a table of many pages
    rows, group, d, ptok = 40, 16, 64, 256
    own = torch.cat([_scores(e, 1, 40, e) for e in (30, 45, 4, 60, 26, 33, 2) * 2])[:rows]
    for e, sign in ((33, 1), (30, -1), (40, 1)):
        _far(kind, d, own, group=group, prefix=_scores(e, sign, 50000, e)[:1], ptok=ptok,
             share=[0] * rows, seed=e)
