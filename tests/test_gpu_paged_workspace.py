"""Workspaces that PagedKV has outgrown: kept, as graphs may hold calls that use them,
but not one for every table that was longer than the last."""
import torch

import pytest

from paper_2605_20600_amd.paged import PagedKV

pytestmark = pytest.mark.gpu


def _growing():
    """A cache, and lists in tables of ever more pages, all of the same tokens."""
    heads, d, ptok = 16, 128, 32
    c = PagedKV("bf16", d, heads, 6 * heads, page_tokens=ptok, group=16)
    g = torch.Generator().manual_seed(1)
    pages = torch.arange(6 * heads, dtype=torch.int32).view(1, heads, 6).cuda()
    k, v = (torch.randn((1, 190, heads, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    c.write(c.lists(pages, None, max_len=0), k, v)
    n = torch.full((1, heads), 190, dtype=torch.int32).cuda()
    q = torch.randn((1, heads * 16, d), generator=g).to(torch.bfloat16).cuda()

    def lists(per):
        table = torch.full((1, heads, per), -1, dtype=torch.int32, device="cuda")
        table[..., :6] = pages
        return c.lists(table, n, max_len=190)
    return c, q, lists


def test_tables_that_grow():
    c, q, lists = _growing()
    want = c.attn(lists(6), q)
    for per in range(1000, 20000, 500):
        assert torch.equal(c.attn(lists(per), q), want)
    kept = sum(t.numel() for t in c._replaced)
    assert len(c._replaced) > 1 and kept <= c._ws.numel()
    # and what is in use is at most twice what the largest table needs
    fresh, q, lists = _growing()
    fresh.attn(lists(per), q)
    assert c._ws.numel() <= 2 * fresh._ws.numel()


def test_a_graph_of_an_outgrown_workspace():
    c, q, lists = _growing()
    small, large = lists(1000), lists(9000)
    want = c.attn(small, q)
    ws = c._ws
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.attn(small, q)
    assert torch.equal(c.attn(large, q), want)
    assert any(t is ws for t in c._replaced)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(c.attn(large, q), want)
