"""The order in which attention starts lists: sorted, left as it is, or another's."""
import pytest
import torch

from test_gpu_paged import LENS, Setup

pytestmark = pytest.mark.gpu


def test_orders_change_nothing():
    s = Setup("int8", 128, 4, LENS, seed=3)
    l = s.lists[0]
    q = s.q.cuda()
    want = s.c.attn(l, q)
    assert l.order is not None and l.order.dtype == torch.int32
    left = s.c.lists(l.pages, l.length, max_len=300, order=False)
    assert left.order is None and left.arg.order is None
    other = s.c.lists(l.pages, l.length, max_len=300, order=l)
    assert other.order is l.order and other.arg.order == l.order.data_ptr()
    # that of lists with other lengths, and of some that have none
    stale = s.c.lists(l.pages, 300 - l.length, max_len=300)
    none = s.c.lists(l.pages, None, max_len=0)
    for x in (left, other, s.c.lists(l.pages, l.length, max_len=300, order=stale),
              s.c.lists(l.pages, l.length, max_len=300, order=none)):
        assert torch.equal(s.c.attn(x, q), want)


def test_refusals():
    s = Setup("int8", 128, 4, LENS, seed=3)
    l = s.lists[0]
    one = s.c.lists(l.pages[:1].contiguous(), l.length[:1].contiguous(), max_len=300)
    for order in (one, True, l.order, 0.5):
        with pytest.raises(ValueError):
            s.c.lists(l.pages, l.length, max_len=300, order=order)
