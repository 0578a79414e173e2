"""Paged attention where its rule on sizes chooses a wavefront for each own list; bounds as
in test_gpu_paged.py."""
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
