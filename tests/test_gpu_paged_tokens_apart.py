"""Attention of several new tokens where values that some of them attend are no finite
numbers: the tokens that do not attend them get the bits they get where all is finite, the
others NaN or an infinity in the dims of such a value (INT8: in all, FP4: in its 32) and
their bits of the finite case in the others.  Beside keys that are none the former are held to
twice the bound of test_gpu_paged.py (its head derives it).

A kernel computes many tokens of a row at once, some of which do not attend the later
ones, or, behind a window, the earlier ones; a weight of 0 times a NaN is one.
"""
import math

import pytest
import torch

from test_gpu_paged import TYPES, U, _reference, _values
from test_gpu_paged_tokens import Case

pytestmark = pytest.mark.gpu
ODD = (math.inf, math.nan, -math.inf)


def _write(c, r, h, t, k, v):
    """Token t of list (r, h) alone."""
    only = torch.full((1,) + tuple(c.table.shape[1:]), -1, dtype=torch.int32)
    only[0, h] = c.table[r, h].cpu()
    heads, d = c.shape[2], c.shape[4]
    lists = c.cache.lists(only.cuda(), None, max_len=t + 1, extra=t)
    c.cache.write(lists, *(x.expand(1, 1, heads, d).contiguous().cuda() for x in (k, v)))


def _run(c):
    rows, tokens, heads, group, d = c.shape
    out = torch.full((rows, tokens, heads * group, d), 7.0, device="cuda")
    lse = torch.full((rows, tokens, heads * group), 7.0, device="cuda")
    c.run(out=out, lse=lse)
    return out.cpu().view(rows, tokens, heads, group, d), lse.cpu().view(rows, tokens, heads, group)


def _check(kind, d, lens, tokens, where, seed=0, **kw):
    """where: [(row, head, token of the list, keys too)], the odd tokens."""
    c = Case(kind, d, lens, tokens, seed=seed, **kw)
    clean, clean_lse = _run(c)
    assert bool(clean.isfinite().all())
    shape = c.k.shape
    k, v = (_values(shape, seed + i, 0.7) for i in (1, 2))  # as Case has them
    rows, _, heads, group, _ = c.shape
    odd = torch.zeros((rows, tokens, heads, d), dtype=torch.bool)  # outputs that are none
    no_key = torch.zeros((rows, tokens, heads), dtype=torch.bool)
    touched = set()
    for n, (r, h, t, keys) in enumerate(where):
        dim = (5 * n + 3) % d
        row_k, row_v = k[r, t, h], v[r, t, h]  # (a token named twice has both)
        row_v[dim] = ODD[n % 3]
        if keys:
            row_k[(7 * n) % d] = ODD[(n + 1) % 3]
        _write(c, r, h, t, row_k, row_v)
        base = int(c.lens[r, h])
        for i in range(max(0, min(c.counts[r], tokens))):
            w = 0 if c.windows is None else int(c.windows[r, h])
            lo = 0 if c.first is None else int(c.first[r, h])
            if w > 0:
                lo = max(lo, base + i + 1 - w)
            if lo <= t <= base + i:
                touched.add((r, i, h))
                dims = dict(bf16=slice(dim, dim + 1), int8=slice(0, d),
                            fp4=slice(dim // 32 * 32, dim // 32 * 32 + 32))[kind]
                odd[r, i, h, dims] = True
                no_key[r, i, h] |= keys
    got, lse = _run(c)
    assert not bool(got[odd[:, :, :, None].expand_as(got)].isfinite().any())
    # (a key that is infinite in one dim may have a score of -inf, so a weight of 0, and leave
    # the value's other dims alone: there is no finite case to compare with)
    mask = (odd | no_key[..., None])[:, :, :, None].expand_as(got)
    off = torch.where(mask, 0, got - clean).abs()
    gone = no_key[..., None].expand_as(lse)
    off_lse = torch.where(gone, 0, torch.where(lse == clean_lse, 0, lse - clean_lse)).abs()
    # a list with an odd key: a column's score of +inf makes the others take another reference
    # too, so that they are as exact, not the same bits
    for r, h in {(r, h) for r, h, _, keys in where if keys}:
        k, v = c.k[r], c.v[r]
        if c.prefix is not None and 0 <= c.share[r] < c.prefix.shape[0]:
            k, v = torch.cat((c.pk[c.share[r]], k)), torch.cat((c.pv[c.share[r]], v))
        k, v, q = k[:, h:h + 1], v[:, h:h + 1], c.q[r].double().view(-1, heads, group, d)[:, h]
        tol, tol_lse = _reference(q.reshape(1, -1, d), k, v, torch.ones((1, len(k)),
                                                                        dtype=torch.bool))[2:]
        assert float(off[r, :, h].max()) <= 2 * tol
        most = float(torch.where(gone[r, :, h], 0, clean_lse[r, :, h]).abs().max())
        assert float(off_lse[r, :, h].max()) <= 2 * (tol_lse + most * U)
        off[r, :, h] = 0
        off_lse[r, :, h] = 0
    assert not bool((off != 0).any()) and not bool((off_lse != 0).any())
    # some of a row's tokens attend one and some do not
    r, h, *_ = where[0]
    seen = sum((r, i, h) in touched for i in range(tokens))
    assert 0 < seen < max(0, min(c.counts[r], tokens))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens", ((64, 1, 2), (128, 1, 5), (128, 3, 5), (64, 1, 16),
                                            (128, 16, 2), (64, 4, 40)))
@pytest.mark.parametrize("keys", (False, True))
def test_a_later_token(kind, d, group, tokens, keys):
    # the last new token, and one in the middle of another head; steps of 32 that begin
    # anywhere among the new tokens
    lens = [[0, 31, 29], [63, 64, 200], [33, 95, 1]]
    last = tokens - 1
    where = [(0, 0, last, keys), (0, 1, 31 + tokens // 2, keys), (1, 0, 63 + last, keys),
             (1, 2, 200 + last, keys), (1, 2, 200 + (tokens + 1) // 2, keys), (2, 1, 95 + last, keys)]
    _check(kind, d, lens, tokens, where, group=group, seed=d + tokens)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens,window", ((128, 1, 5, 40), (64, 2, 8, 3), (64, 1, 33, 70)))
def test_a_token_behind_a_window(kind, d, group, tokens, window):
    lens = [[100, 133], [97, 64]]
    windows = [[window, 0], [window, window]]
    half = tokens // 2
    where = [(0, 0, 100 + half + 1 - window, False), (1, 0, 97 + 1 - window, False),
             (1, 1, 64 + half + 1 - window + (window < 5), True)]
    _check(kind, d, lens, tokens, where, group=group, windows=windows, seed=3)
    # and with a first token of the list between them, and rows that have fewer tokens
    first = [[100 + half - window, 0], [0, 20]]
    _check(kind, d, lens, tokens, where + [(0, 1, 133 + tokens - 2, False)], group=group,
           windows=windows, first=first, counts=[tokens - 1, tokens], seed=4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group,tokens,rows", ((1, 5, 9), (4, 3, 12)))
def test_with_a_shared_prefix(kind, group, tokens, rows):
    lens = torch.randint(0, 130, (rows, 2), generator=torch.Generator().manual_seed(rows)).tolist()
    share = [(0, -1, 1)[i % 3] for i in range(rows)]
    where = [(r, r % 2, lens[r][r % 2] + tokens - 1 - r % 2, r % 4 == 3) for r in range(rows)]
    _check(kind, 128, lens, tokens, where, group=group, prefix=[[333, 64], [31, 1025]], share=share,
           seed=2)


@pytest.mark.parametrize("kind", TYPES)
def test_lists_of_several_parts(kind):
    lens = [[5001], [4090]]
    where = [(0, 0, 5003, False), (1, 0, 4090, False), (1, 0, 4093, True), (1, 0, 4094, False)]
    _check(kind, 128, lens, 5, where, group=2, seed=9)


@pytest.mark.parametrize("kind", TYPES)
def test_many_short_lists(kind):
    # a wavefront a list
    lens = torch.randint(0, 20, (350, 2), generator=torch.Generator().manual_seed(12)).tolist()
    where = [(r, 1, lens[r][1] + 1 + r % 2, r % 5 == 0) for r in range(0, 350, 7)]
    _check(kind, 64, lens, 3, where, seed=12)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens,most", ((128, 4, 64, 9000), (64, 1, 130, 15000)))
def test_pieces_of_prompts(kind, d, group, tokens, most):
    # cuts of 128 columns, planned on the device: a later token of the same wavefront's columns,
    # of another's and of another cut; behind windows; lists of several chunks and of one
    lens = [[most, 130], [97, most // 3], [5, 0]]
    windows = [[0, 64], [0, 300], [0, 0]]
    where = [(0, 0, most + tokens // 2, False), (0, 0, most + 3, False), (0, 1, 130 + 9 - 64, False),
             (0, 1, 130 + tokens - 1, True), (1, 1, most // 3 + 40 - 300, False),
             (2, 0, 5 + 17, False), (2, 1, tokens - 1, False)]
    _check(kind, d, lens, tokens, where, group=group, ptok=256, windows=windows, seed=24)
    _check(kind, d, lens, tokens, where, group=group, ptok=256, windows=windows,
           counts=[tokens, tokens, 30], prefix=[[70, 600]], share=[0, -1, 0], seed=25)


@pytest.mark.parametrize("kind", TYPES)
def test_many_cuts_of_many_columns(kind):
    # a block a cut
    lens = torch.randint(0, 90, (65, 4), generator=torch.Generator().manual_seed(26)).tolist()
    lens[3] = [2300, 10, 2048, 0]
    where = [(3, 0, 2300 + 64, False), (3, 2, 2048 + 128, False), (3, 2, 2048 + 129, False)]
    where += [(r, r % 4, lens[r][r % 4] + (31 * r) % 129 + 1, r % 9 == 0) for r in range(4, 65, 3)]
    _check(kind, 64, lens, 130, where, windows=[[0, 30, 2200, 0]] * 65, seed=26)


def test_values_too_large_for_four_bits():
    # finite bf16 that FP4 rounds up to 2^128
    c = Case("fp4", 64, [[40], [3]], 4, group=2, seed=5)
    clean, _ = _run(c)
    v = _values(c.k.shape, 7, 0.7)
    row = v[0, 42, 0].clone()
    row[9] = torch.finfo(torch.bfloat16).max
    _write(c, 0, 0, 42, _values(c.k.shape, 6, 0.7)[0, 42, 0], row)
    got, _ = _run(c)
    assert torch.equal(got[1], clean[1]) and torch.equal(got[0, :2], clean[0, :2])
    assert not bool(got[0, 2:, :, :, 9].isfinite().any())
    assert torch.equal(got[0, 2:, ..., 32:], clean[0, 2:, ..., 32:])
