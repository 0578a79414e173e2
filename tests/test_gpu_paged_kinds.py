"""Paged attention where its rules on sizes choose a wavefront for each own list, or
blocks of 256 columns for a prefix; bounds as in test_gpu_paged.py."""
import pytest
import torch

from test_gpu_paged import TYPES, Setup, _short_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group", ((64, 1), (64, 5), (128, 1), (128, 16)))
def test_a_wavefront_for_a_list(kind, d, group):
    # 110 x 16 lists of up to 100 tokens
    s = Setup(kind, d, 16, _short_lists(110, 16, 100, d + group), ptok=32, group=group, seed=61)
    s.check()
    first = torch.randint(-3, 110, (110, 16), generator=torch.Generator().manual_seed(1))
    first[2] = 2 ** 31 - 1
    s.check(first=first.tolist())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,group", ((64, 1), (64, 3), (64, 7), (128, 2)))
def test_a_wavefront_for_a_list_beside_prefixes(kind, d, group):
    # in the order of the launch, rows of two prefixes, of one without tokens and of none
    g = torch.Generator().manual_seed(group)
    rows, heads = 26, 50
    prefix = torch.randint(0, 1400, (3, heads), generator=g)
    prefix[2] = 0
    s = Setup(kind, d, heads, _short_lists(rows, heads, 80, 9), group=group, seed=63,
              prefix_lens=prefix.tolist())
    share = torch.randint(-1, 4, (rows,), generator=g).tolist()  # (3 is no list)
    share[0], share[1] = 0, 0
    s.check(share=share)
    first = torch.randint(0, 60, (rows, heads), generator=g).tolist()
    s.check(share=[1] * rows, first=first,
            shared_first=torch.randint(0, 900, (3, heads), generator=g).tolist())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,ptok,group,rows", ((128, 64, 16, 43), (64, 32, 7, 60), (128, 256, 2, 180),
                                              (64, 64, 13, 41), (128, 32, 1, 520)))
def test_blocks_of_many_columns(kind, d, ptok, group, rows):
    # tables of 90000 tokens: work for blocks of 256 columns for every type, if all were there
    g = torch.Generator().manual_seed(rows)
    lens = torch.randint(0, 60, (rows, 2), generator=g).tolist()
    s = Setup(kind, d, 2, lens, ptok=ptok, group=group, prefix_lens=[[4400, 97], [290, 0]], seed=d + 1)
    l = s.lists[1]
    table = torch.full((2, 2, -(-90000 // ptok)), -1, dtype=torch.int32).cuda()
    table[:, :, :l.pages.shape[2]] = l.pages
    s.lists[1] = s.c.lists(table, l.length, max_len=90000)
    share = [(0, 0, 1, -1, 0)[i % 5] for i in range(rows)]
    s.check(share=share)
    s.check(share=[0] * (rows - 1) + [1])
    for i, (b, h, p) in enumerate(((0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1))):
        s.lists[1].pages[b, h, p] = (-1, s.c.cfg.num_pages, -7)[i]
    s.check(share=share, shared_first=[[1003, 96], [31, 5]],
            shared_dropped=[(0, 0, 0), (0, 0, 3000 // ptok), (1, 0, 1)])
