"""Attention of several new tokens of each row over a paged cache against a plain 64-bit
implementation, with the bounds of test_gpu_paged.py (its head derives them).

Every pool is filled with bytes 255 first (NaN as bf16 and as any scale), so that what was
never written may not be seen; lists and prefixes, windows and dropped pages, tokens that
counts leave out, and pieces that end inside a step are among the cases.
"""
import math

import pytest
import torch

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.paged import PagedKV
from test_gpu_paged import TYPES, U, _cache, _held, _reference, _values

pytestmark = pytest.mark.gpu


class Case:
    """lens: [rows][heads] tokens before the new ones."""

    def __init__(self, kind, d, lens, tokens, counts=None, group=1, ptok=64, windows=None,
                 first=None, prefix=None, share=None, dropped=(), seed=0, extra=0, spare=1):
        g = torch.Generator().manual_seed(seed)
        lens = torch.tensor(lens, dtype=torch.int32)
        rows, heads = lens.shape
        self.shape = rows, tokens, heads, group, d
        self.counts = [tokens] * rows if counts is None else counts
        own_most = int(lens.max()) + tokens
        per = -(-own_most // ptok) + spare
        sizes = [rows * heads * per]
        if prefix is not None:
            prefix = torch.tensor(prefix, dtype=torch.int32)
            pre_per = max(1, -(-int(prefix.max()) // ptok))
            sizes.append(prefix.numel() * pre_per)
        numbers = torch.randperm(sum(sizes) + 5, generator=g).to(torch.int32)
        self.cache = _cache(kind, d, heads, sum(sizes) + 5, page_tokens=ptok, group=group)
        table = numbers[:sizes[0]].view(rows, heads, per).clone()
        for r, h, p in dropped:
            table[r, h, p] = -1
        self.table = table.cuda()
        most = max(1, own_most)
        self.k, self.v = (_values((rows, most, heads, d), seed + i, 0.7) for i in (1, 2))
        start = torch.zeros_like(lens)
        # what is there, then the new tokens behind it
        past = max(1, int(lens.max()))
        for r in range(rows):
            for h in range(heads):
                n = int(lens[r, h]) + max(0, min(self.counts[r], tokens))
                part = self.cache.lists(self.table[r:r + 1, h:h + 1].expand(1, heads, -1)
                                        .contiguous(), None, max_len=0)
                if n:  # one head's tokens alone: the others' rows go to a table of no pages
                    only = torch.full((1, heads, per), -1, dtype=torch.int32)
                    only[0, h] = table[r, h]
                    part = self.cache.lists(only.cuda(), None, max_len=0)
                    self.cache.write(part, self.k[r:r + 1, :n].contiguous().cuda(),
                                     self.v[r:r + 1, :n].contiguous().cuda())
        self.k, self.v = _held(self.k, kind), _held(self.v, kind)
        self.lens, self.dropped, self.ptok = lens, dropped, ptok
        self.first = None if first is None else torch.tensor(first, dtype=torch.int32)
        self.lists = self.cache.lists(self.table, (lens - extra).cuda(), max_len=past,
                                      first=None if first is None else self.first.cuda(),
                                      extra=extra)
        self.windows = None if windows is None else torch.tensor(windows, dtype=torch.int32)
        self.prefix, self.share, self.shared = prefix, share, None
        if prefix is not None:
            n = max(1, int(prefix.max()))
            pk, pv = (_values((prefix.shape[0], n, heads, d), seed + i, 0.7) for i in (3, 4))
            pt = numbers[sizes[0]:sum(sizes)].view(*prefix.shape, -1).cuda()
            self.cache.write(self.cache.lists(pt, None, max_len=0), pk.cuda(), pv.cuda())
            self.pk, self.pv = _held(pk, kind), _held(pv, kind)
            self.shared = self.cache.lists(pt, prefix.cuda(), max_len=int(prefix.max()))
        self.q = (1.3 * torch.randn((rows, tokens, heads * group, d), generator=g)).to(
            torch.bfloat16)
        self.keep = self.lists, self.shared

    def run(self, q=None, out=None, lse=None, counts=True):
        rows, tokens, heads, group, d = self.shape
        c = torch.tensor(self.counts, dtype=torch.int32).cuda() if counts else None
        share = None if self.share is None else torch.tensor(self.share, dtype=torch.int32).cuda()
        return self.cache.attn_tokens(
            self.lists, self.q.cuda() if q is None else q, counts=c,
            window=None if self.windows is None else self.windows.cuda(), shared=self.shared,
            share=share, out=out, lse=lse)

    def check(self, q=None):
        rows, tokens, heads, group, d = self.shape
        hq = heads * group
        last = None
        for _ in range(2):  # the workspace is left as it was found
            out = torch.full((rows, tokens, hq, d), 7.0, device="cuda")
            lse = torch.full((rows, tokens, hq), 7.0, device="cuda")
            self.run(q, out, lse)
            assert last is None or torch.equal(out, last), "not deterministic"
            last = out
        got, got_lse = out.cpu().double(), lse.cpu().double()
        capacity = self.table.shape[2] * self.ptok
        for r in range(rows):
            n = max(0, min(self.counts[r], tokens))
            assert bool((got[r, n:] == 7).all()) and bool((got_lse[r, n:] == 7).all())
            at = torch.arange(self.k.shape[1])
            for i in range(n):
                end = (self.lens[r] + i + 1).clamp(max=capacity)
                lo = torch.zeros_like(end) if self.first is None else self.first[r].clone()
                if self.windows is not None:
                    w = self.windows[r]
                    lo = torch.where(w > 0, torch.maximum(lo, self.lens[r] + i + 1 - w), lo)
                seen = (at < end[:, None]) & (at >= lo[:, None])
                for dr, dh, dp in self.dropped:
                    if dr == r:
                        seen[dh, dp * self.ptok:(dp + 1) * self.ptok] = False
                k, v = self.k[r], self.v[r]
                j = -1 if self.share is None else self.share[r]
                if self.share is not None and 0 <= j < self.prefix.shape[0]:
                    ps = torch.arange(self.pk.shape[1]) < self.prefix[j][:, None]
                    k, v = torch.cat((self.pk[j], k)), torch.cat((self.pv[j], v))
                    seen = torch.cat((ps, seen), 1)
                ref, ref_lse, tol, tol_lse = _reference(
                    self.q[r, i].double().view(heads, group, d), k, v, seen)
                ref, ref_lse = ref.reshape(hq, d), ref_lse.reshape(hq)
                err = float((got[r, i] - ref).abs().max())
                assert err <= tol, (r, i, err, tol)
                empty = ref_lse == -math.inf
                assert torch.equal(got_lse[r, i] == -math.inf, empty)
                assert not got[r, i][empty].any()
                off = (got_lse[r, i] - ref_lse)[~empty].abs()
                assert bool((off <= tol_lse + ref_lse[~empty].abs() * U).all()), (r, i)


LENS = [[0, 1, 31, 32], [33, 63, 64, 65], [200, 127, 3, 0], [96, 95, 300, 129]]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens", ((64, 1, 1), (64, 3, 5), (128, 1, 5), (128, 1, 16),
                                            (128, 2, 9), (64, 1, 33), (128, 16, 2), (128, 5, 4),
                                            (64, 7, 8)))
def test_ragged_lists(kind, d, group, tokens):
    Case(kind, d, LENS, tokens, group=group, seed=d + tokens).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group,tokens", ((1, 6), (4, 19)))
def test_counts(kind, group, tokens):
    Case(kind, 64, LENS, tokens, counts=[3, 0, tokens + 9, -4], group=group, seed=1).check()
    Case(kind, 64, LENS, tokens, counts=[0, 0, 0, 0], group=group, seed=1).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ptok,group,tokens", ((32, 1, 7), (64, 2, 40), (256, 3, 5)))
def test_windows_firsts_and_dropped_pages(kind, ptok, group, tokens):
    lens = [[700, 513, 512, 511], [40, 700, 1, 650]]
    windows = [[1, 0, 98, 33], [64, -5, 7, 2 ** 31 - 1]]
    Case(kind, 128, lens, tokens, group=group, ptok=ptok, windows=windows, seed=5).check()
    first = [[0, 500, 512, 100], [39, 650, 1, 31]]
    Case(kind, 128, lens, tokens, group=group, ptok=ptok, windows=windows, first=first,
         dropped=[(0, 0, 0), (0, 1, 512 // ptok), (1, 3, 0), (1, 1, 600 // ptok),
                  (1, 0, 40 // ptok)], seed=6).check()
    # lists of which a first leaves the earliest tokens nothing
    Case(kind, 128, [[10, 20], [30, 0]], tokens, group=group, ptok=ptok,
         first=[[12, 2 ** 31 - 1], [31, 3]], seed=7).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens,rows", ((128, 1, 5, 9), (64, 4, 3, 12), (128, 3, 17, 5),
                                                (64, 1, 4, 90)))
def test_shared_prefixes(kind, d, group, tokens, rows):
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 130, (rows, 2), generator=g).tolist()
    share = [(0, 2, 0, -1, 1, 0, 3)[i % 7] for i in range(rows)]
    counts = [(tokens, 1, tokens, 0, 2)[i % 5] for i in range(rows)]
    prefix = [[333, 64], [0, 0], [31, 1025]]
    Case(kind, d, lens, tokens, group=group, prefix=prefix, share=share, seed=2).check()
    Case(kind, d, lens, tokens, counts=counts, group=group, prefix=prefix, share=share,
         windows=[[0, 20]] * rows, seed=3).check()
    Case(kind, d, lens, tokens, group=group, prefix=prefix, share=[-1] * rows, seed=4).check()


@pytest.mark.parametrize("kind,heads,group,tokens,rows,most", (
    ("bf16", 2, 4, 3, 65, 8192), ("int8", 2, 8, 2, 65, 16384), ("fp4", 4, 16, 1, 65, 16384)))
def test_prefixes_of_many_columns(kind, heads, group, tokens, rows, most):
    # prefixes that blocks of 256 columns take
    prefix = [[most] + [most - 97] * (heads - 1)]
    Case(kind, 128, [[40, 3, 0, 9][:heads]] * rows, tokens, group=group, prefix=prefix,
         share=[0] * (rows - 1) + [-1], counts=[tokens] * (rows - 2) + [0, tokens], ptok=256,
         seed=8).check()


@pytest.mark.parametrize("kind", TYPES)
def test_long_lists_in_chunks(kind):
    # parts of several blocks, joined by the last; long pieces of a prompt
    Case(kind, 128, [[5001], [4090], [17]], 5, group=2, seed=9).check()
    Case(kind, 64, [[2040], [0]], 70, group=3, windows=[[0], [30]], seed=10).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens", ((128, 1, 300), (64, 3, 90), (128, 7, 37), (64, 16, 33)))
def test_pieces_of_prompts(kind, d, group, tokens):
    # cuts of many columns: of one chunk and of several, windows that begin inside them,
    # rows that end before a cut does or have none, prefixes, dropped pages
    counts = [tokens, tokens // 2, 1, 0]
    lens = [[0, 130], [97, 31], [5, 0], [3, 4]]
    Case(kind, d, lens, tokens, counts=counts, group=group, seed=20).check()
    Case(kind, d, lens, tokens, counts=counts, group=group, windows=[[50, 7], [0, 64]] * 2,
         first=[[3, 33], [0, 90], [6, 0], [0, 0]], dropped=[(0, 1, 1), (1, 0, 0)], seed=21).check()
    Case(kind, d, lens, tokens, counts=counts, group=group, prefix=[[70, 600], [0, 0]],
         share=[0, 1, 0, 0], seed=22).check()
    Case(kind, d, [[1500, 1030]], tokens, group=group, ptok=256, windows=[[0, 900]], seed=23).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group,tokens,most", ((128, 4, 64, 9000), (64, 1, 130, 15000)))
def test_pieces_of_prompts_behind_long_lists(kind, d, group, tokens, most):
    # cuts of 128 columns (their work is enough): lists of several pieces of 2048 tokens and
    # of a few tokens, in chunks of a length that follows from all of them
    counts = [tokens, tokens - 1, 7, 0]
    lens = [[most, 130], [97, most // 3], [5, 0], [3, 4]]
    Case(kind, d, lens, tokens, counts=counts, group=group, ptok=256, seed=24).check()
    Case(kind, d, lens, tokens, counts=counts, group=group, windows=[[2100, 7], [0, 64]] * 2,
         first=[[3, 33], [0, 2050], [6, 0], [0, 0]], dropped=[(0, 0, 40), (0, 0, 33), (1, 0, 0)],
         prefix=[[70, 600], [0, 0]], share=[0, 1, -1, 0], seed=25).check()


@pytest.mark.parametrize("kind", TYPES)
def test_more_cuts_than_are_planned_together(kind):
    # 513 cuts of 128 columns and more, each a block's; lists of more than 2048 tokens
    g = torch.Generator().manual_seed(26)
    lens = torch.randint(0, 90, (65, 4), generator=g).tolist()
    lens[3] = [2300, 10, 2048, 0]
    counts = [(130, 64, 1, 0, 129)[i % 5] for i in range(65)]
    Case(kind, 64, lens, 130, counts=counts, group=1, windows=[[0, 30, 2200, 0]] * 65,
         seed=26).check()


@pytest.mark.parametrize("kind", TYPES)
def test_a_prompt_from_nothing(kind):
    Case(kind, 128, [[0, 0]] * 3, 100, counts=[100, 33, 1], group=2, seed=11).check()


def test_many_short_lists():
    # where a wavefront takes a list, not a block
    g = torch.Generator().manual_seed(12)
    lens = torch.randint(0, 20, (350, 2), generator=g).tolist()
    Case("int8", 64, lens, 3, seed=12).check()
    Case("int8", 64, lens, 3, prefix=[[40, 7]], share=[i % 2 - 1 for i in range(350)],
         seed=13).check()


def test_bounds_and_tables_that_end():
    # a table that ends before the last new tokens: they were not stored, and are not seen
    Case("bf16", 64, [[60, 40]], 8, spare=0, seed=14).check()
    Case("int8", 64, [[62, 30]], 40, ptok=32, spare=-1, seed=15).check()
    # lengths that the host counts in part
    Case("fp4", 64, [[100, 70], [9, 33]], 6, extra=9, windows=[[0, 12]] * 2, seed=16).check()


def test_queries_of_any_stride():
    c = Case("int8", 128, [[50, 3], [0, 200]], 6, group=2, seed=17)
    rows, tokens, heads, group, d = c.shape
    hq = heads * group
    wide = torch.full((rows, tokens, 3 * hq * d + 8), math.nan, dtype=torch.bfloat16,
                      device="cuda")
    part = wide[..., hq * d:2 * hq * d].unflatten(2, (hq, d))
    part.copy_(c.q)
    c.check(part)
    turned = torch.full((tokens, rows, hq, d), math.nan, dtype=torch.bfloat16, device="cuda")
    turned.copy_(c.q.transpose(0, 1))
    c.check(turned.transpose(0, 1))
    # the same token's queries for all
    c.q = c.q[:, :1].expand(-1, tokens, -1, -1)
    c.check(c.q[:, :1].cuda().expand(-1, tokens, -1, -1))


def test_one_token_as_the_call_of_one_query():
    c = Case("int8", 128, LENS, 1, group=3, seed=18)
    out = c.run()
    one = c.cache.lists(c.table, (c.lens + 1).cuda(), max_len=301)
    assert torch.equal(out[:, 0], c.cache.attn(one, c.q[:, 0].contiguous().cuda()))


def test_replays_and_streams():
    c = Case("int8", 64, [[40, 700], [0, 33]], 4, group=2, prefix=[[300, 20]], share=[0, 0],
             seed=19)
    q = c.q.cuda()
    counts = torch.tensor([4, 3], dtype=torch.int32).cuda()
    share = torch.zeros(2, dtype=torch.int32).cuda()
    out = torch.zeros((2, 4, 4, 64), device="cuda")

    def call():
        return c.cache.attn_tokens(c.lists, q, counts=counts, shared=c.shared, share=share,
                                   out=out)
    eager = call().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        q.copy_((1.3 * torch.randn(q.shape, generator=torch.Generator().manual_seed(i))).bfloat16())
        out.zero_()
        want = call().clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals():
    c = Case("int8", 64, [[4, 5]], 2)
    q = c.q.cuda()
    ok = torch.zeros(1, dtype=torch.int32, device="cuda")
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()), dict(q=q[:, :, :1]),
               dict(q=q.transpose(2, 3)), dict(counts=ok.long()), dict(counts=ok.cpu()),
               dict(window=ok), dict(share=ok[:0]), dict(out=q), dict(lse=q),
               dict(own=PagedKV("int8", 64, 1, 5).lists(c.table[:, :1].contiguous(), None, 0))):
        with pytest.raises(ValueError):
            c.cache.attn_tokens(**{"own": c.lists, "q": q, **kw})
    with pytest.raises(B.HeadKVError):
        c.cache.attn_tokens(c.lists, q, share=ok)
    assert c.cache.attn_tokens(c.lists, q[:, :0]).shape == (1, 0, 2, 64)
