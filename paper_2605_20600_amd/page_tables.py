"""Page tables, lengths and windows of many rows and layers, brought from one step to the
next on the GPU: what a row has gained may be known there alone.

PyTorch supplies device memory and the stream, as for Session; the computation is a
call into libheadkv.so through the binding.  Calls are made on the current device and
its current stream; tensors that lie elsewhere are refused.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .paged import Lists, _device_int32, _stream
from .session import _ptr


class PageTables:
    """The lists of `rows` rows in each of `layers` layers, whose pages come from one pool
    (or one pool for each layer's caches of num_pages pages in all), and the ring of free
    pages.  `pages` [layers * rows][kv_heads][max_pages], `len`, `first` [layers * rows]
    [kv_heads], `order` [layers][rows * kv_heads], `free_pages` [num_pages] and `free_state`
    [4] (place and number of the free pages; pages that the last extend() lacked) are views
    of `buffer`, int32, which is all the state there is.  Use one per stream."""

    def __init__(self, kv_heads: int, max_pages: int, num_pages: int, rows: int, layers: int = 1,
                 page_tokens: int = 64, window: Optional[torch.Tensor] = None,
                 device: str = "cuda"):
        """window: int32 [layers * rows][kv_heads], tokens that the next token of a list
        attends, itself among them; 0: all."""
        lists = layers * rows
        n = lists * kv_heads
        arg = B.PagedTablesArg(None, None, None, None, None, None, None, kv_heads, page_tokens,
                               num_pages, lists, rows, max_pages)
        need = B.headkv_paged_extend_plan(arg)
        sizes = (n * max_pages, n, n, n, num_pages, 4)
        self.buffer = torch.zeros(sum(sizes), dtype=torch.int32, device=device)
        self.index = self.buffer.get_device()
        pages, length, first, order, self.free_pages, self.free_state = \
            self.buffer.split_with_sizes(sizes)
        self.pages = pages.view(lists, kv_heads, max_pages)
        self.len, self.first = (t.view(lists, kv_heads) for t in (length, first))
        self.order = order.view(layers, rows * kv_heads)
        self.pages.fill_(-1)
        torch.arange(num_pages, out=self.free_pages)
        self.order[:] = torch.arange(rows * kv_heads, device=device)
        self.free_state[1] = num_pages
        if window is not None:
            _device_int32(window, (lists, kv_heads), "window", self.index)
        self.window = window
        self.rows, self.layers, self.capacity = rows, layers, max_pages * page_tokens
        self._ws = torch.empty(need, dtype=torch.uint8, device=device)
        for name, t in (("pages", self.pages), ("len", self.len), ("first", self.first),
                        ("order", self.order), ("window", window),
                        ("free_pages", self.free_pages), ("free_state", self.free_state)):
            setattr(arg, name, _ptr(t))
        self.arg = arg

    def lists(self, layer: int = 0, max_len: Optional[int] = None) -> Lists:
        """A layer's lists, as they are whenever a call uses them; max_len: no list gets
        longer (None: than its table)."""
        if not 0 <= layer < self.layers:
            raise ValueError(f"layer {layer} of {self.layers}")
        at = slice(layer * self.rows, (layer + 1) * self.rows)
        got = Lists(self.pages[at], self.len[at], self.capacity if max_len is None else max_len,
                    first=self.first[at], order=False)
        got.order = self.order[layer]  # as extend() has left it
        got.arg.order = _ptr(got.order)
        return got

    def extend(self, tokens: int, advance: Optional[torch.Tensor] = None,
               counts: Optional[torch.Tensor] = None) -> None:
        """Before the next `tokens` tokens (counts: int32 [rows], of each row) are written:
        lists grow by `advance` (int32 [rows], what each row has gained since the last call;
        negative: its lists end), windows move on, pages behind them become free, and pages
        for the tokens to come are taken."""
        if advance is not None:
            _device_int32(advance, (self.rows,), "advance", self.index)
        if counts is not None:
            _device_int32(counts, (self.rows,), "counts", self.index)
        B.headkv_paged_extend(self.arg, _ptr(advance), _ptr(counts), tokens, self._ws.data_ptr(),
                              self._ws.numel(), _stream(self.index))
