"""Paged attention beside tokens that are NaN: past every list's own length and before
its window, as a page in use holds what another sequence left there.  The checks and
bounds of test_gpu_paged.py."""
import math

import pytest
import torch

from test_gpu_paged import LENS, TYPES, Setup, _short_lists

pytestmark = pytest.mark.gpu


class Tails(Setup):
    """Lists whose tokens past their length, up to the page's end and further, are NaN."""

    def __init__(self, *args, first=None, shared_first=None, **kw):
        super().__init__(*args, **kw)
        self.first, self.shared_first = first, shared_first
        for l, before in zip(self.lists, (first, shared_first)):
            nan = torch.full((l.n, 300, l.kv_heads, self.c.head_dim), math.nan,
                             dtype=torch.bfloat16, device="cuda")
            self.c.write(l, nan, nan)  # behind each head's own length
            if before is None:
                continue
            before = torch.tensor(before, dtype=torch.int32).cuda()
            for i in range(1, 40):  # and just before its window
                there = before >= i
                pages = torch.where(there[..., None], l.pages, -1).contiguous()
                at = torch.minimum(torch.where(there, before - i, 0), l.length).contiguous()
                self.c.write(self.c.lists(pages, at, max_len=l.arg.max_len), nan[:, :1], nan[:, :1])

    def check(self, **kw):
        super().check(first=self.first, shared_first=self.shared_first, **kw)


@pytest.mark.parametrize("kind", TYPES)
def test_the_tails_are_nan(kind):
    # each list one token longer than it is sees one of them
    s = Tails(kind, 64, 4, LENS)
    longer = (s.lens[0] + 1).cuda()
    got = s.c.attn(s.c.lists(s.lists[0].pages, longer, max_len=400), s.q.cuda())
    assert bool(got.isnan().all())
    k, v = s.c.read(s.c.lists(s.lists[0].pages, longer, max_len=400), 1, begin=-1)
    assert bool(k.isnan().all()) and bool(v.isnan().all())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("ptok,group", ((32, 1), (64, 3), (256, 16)))
def test_ragged_lists(kind, d, ptok, group):
    Tails(kind, d, 4, LENS, ptok=ptok, group=group, seed=d + group).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ptok", (32, 256))
def test_windows(kind, ptok):
    Tails(kind, 128, 4, [[700, 513, 512, 511], [40, 700, 1, 650]], ptok=ptok, group=2, seed=5,
          first=[[3, 500, 512, 100], [39, 650, 1, 31]]).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", (64, 128))
def test_many_short_lists(kind, d):
    Tails(kind, d, 16, _short_lists(110, 16, 100, d), ptok=32, seed=61).check()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("group,rows", ((1, 5), (4, 37), (16, 20)))
def test_prefixes(kind, group, rows):
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 130, (rows, 2), generator=g).tolist()
    s = Tails(kind, 128, 2, lens, group=group, prefix_lens=[[333, 64], [0, 0], [31, 1025]],
              shared_first=[[40, 63], [0, 0], [0, 1000]], seed=group)
    s.check(share=[(0, 2, 0, -1, 1, 0, 3)[i % 7] for i in range(rows)])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,ptok,group,rows", ((128, 64, 16, 43), (64, 32, 13, 41)))
def test_blocks_of_many_columns(kind, d, ptok, group, rows):
    # tables of 90000 tokens: work for blocks of 256 columns, if all were there
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 60, (rows, 2), generator=g).tolist()
    s = Tails(kind, d, 2, lens, ptok=ptok, group=group, prefix_lens=[[4400, 97], [290, 1]], seed=d,
              shared_first=[[1003, 50], [31, 0]])
    l = s.lists[1]
    table = torch.full((2, 2, -(-90000 // ptok)), -1, dtype=torch.int32).cuda()
    table[:, :, :l.pages.shape[2]] = l.pages
    s.lists[1] = s.c.lists(table, l.length, max_len=90000)
    s.check(share=[(0, 0, 1, -1, 0)[i % 5] for i in range(rows)])
