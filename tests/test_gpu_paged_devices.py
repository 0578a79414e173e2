"""Paged calls where several GPUs are in use: nothing is launched unless the cache, every
tensor and the current device are one.  (Other devices are stood in for: the check runs
before anything is launched.)"""
import pytest
import torch

from paper_2605_20600_amd import paged
from paper_2605_20600_amd.paged import PagedKV, token_logprobs

pytestmark = pytest.mark.gpu


def _cache():
    c = PagedKV("bf16", 64, 2, 6, page_tokens=32)
    pages = torch.arange(6, dtype=torch.int32, device="cuda").view(1, 2, 3)
    return c, c.lists(pages, None, max_len=0)


def _rows():
    return torch.ones((1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")


def test_the_device_is_known():
    c, l = _cache()
    assert c.device == torch.device("cuda", torch.cuda.current_device()) and c.pool.device == c.device
    assert l.index == c.index == c.device.index


def test_another_current_device(monkeypatch):
    c, l = _cache()
    rows = _rows()
    c.write(l, rows, rows)
    before = c.pool.clone()
    x = torch.zeros((2, 10), device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros((1, 2, 64), device="cuda")
    monkeypatch.setattr(paged, "_current_device", lambda: c.index + 1)
    for call in (lambda: c.write(l, rows + 1, rows), lambda: c.read(l, 4, k=rows, v=rows.clone()),
                 lambda: c.attn(l, rows[:, 0], out=out), lambda: token_logprobs(x, t)):
        with pytest.raises(ValueError, match="current device"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(c.pool, before) and bool((rows == 1).all()) and not out.any()


def test_a_cache_elsewhere():
    c, l = _cache()
    rows = _rows()
    c.index += 1
    for call in (lambda: c.write(l, rows, rows), lambda: c.read(l, 4, k=rows, v=rows.clone()),
                 lambda: c.attn(l, rows[:, 0]), lambda: c.lists(l.pages, None, max_len=0)):
        with pytest.raises(ValueError):
            call()


def test_lists_elsewhere():
    c, l = _cache()
    rows = _rows()
    share = torch.zeros(1, dtype=torch.int32, device="cuda")
    other = c.lists(l.pages, None, max_len=0)
    other.index += 1
    for call in (lambda: c.write(other, rows, rows), lambda: c.read(other, 4),
                 lambda: c.attn(other, rows[:, 0]),
                 lambda: c.attn(l, rows[:, 0], shared=other, share=share)):
        with pytest.raises(ValueError, match="lists on"):
            call()
