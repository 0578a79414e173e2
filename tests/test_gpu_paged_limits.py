"""Paged attention beside tables of so many prefixes that their blocks take several
launches."""
import pytest
import torch

from paper_2605_20600_amd.paged import PagedKV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefixes", (1 << 13, 1 << 14))
def test_tables_of_very_many_prefixes(prefixes):
    # 2^23 and 2^24 lists: all but two, near the ends of the table, have no page and no
    # tokens, and nobody reads them
    heads, d, ptok, rows = 1024, 64, 32, 3
    c = PagedKV("bf16", d, heads, 5 * heads, page_tokens=ptok)
    g = torch.Generator().manual_seed(prefixes)
    pages = torch.arange(5 * heads, dtype=torch.int32).view(5, heads, 1).cuda()
    lens = torch.randint(1, ptok + 1, (5, heads), generator=g).to(torch.int32).cuda()
    k, v = (torch.randn((5, ptok, heads, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    c.write(c.lists(pages, None, max_len=0), k, v)
    q = torch.randn((rows, heads, d), generator=g).to(torch.bfloat16).cuda()
    own = c.lists(pages[:rows].contiguous(), lens[:rows].contiguous(), max_len=ptok)
    few = c.lists(pages[rows:].contiguous(), lens[rows:].contiguous(), max_len=ptok)
    share = torch.tensor([1, 0, 1], dtype=torch.int32).cuda()
    want = c.attn(own, q, shared=few, share=share)
    table = torch.full((prefixes, heads, 1), -1, dtype=torch.int32, device="cuda")
    length = torch.zeros((prefixes, heads), dtype=torch.int32, device="cuda")
    at = [1, prefixes - 1]
    table[at], length[at] = pages[rows:], lens[rows:]
    many = c.lists(table, length, max_len=ptok)
    share = torch.tensor([at[1], at[0], at[1]], dtype=torch.int32).cuda()
    for _ in range(2):  # the workspace is left as it was found
        got = c.attn(own, q, shared=many, share=share)
        assert torch.equal(got, want)
