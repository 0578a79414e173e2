"""A paged key/value cache of 16, 8 or 4 bits, decode attention over it with
prefixes that rows share, and the scores of sampled tokens.

PyTorch supplies device memory and the stream, as for Session; every
computation is a call into libheadkv.so through the binding.  Calls are made on the
current device and its current stream; tensors that lie elsewhere are refused.
"""
from __future__ import annotations

from functools import lru_cache
from typing import TYPE_CHECKING, Dict, List, Optional, Tuple, Union

import torch

from . import binding as B
from .session import _ptr

if TYPE_CHECKING:
    from .rotary import NormWeights, Rotary


# torch's public calls where a torch has no such private ones, which cost less (see
# Session.stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream(index: int) -> int:
    """The current stream, of device `index`."""
    if _current_device() != index:
        raise ValueError(f"tensors on cuda:{index}, but the current device is "
                         f"cuda:{_current_device()}")
    return _raw_stream(index)


def _device_int32(t: torch.Tensor, shape: Tuple[int, ...], name: str, index: int) -> torch.Tensor:
    if t.dtype != torch.int32 or t.shape != shape or t.get_device() != index or index < 0 \
            or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape} on "
                         f"{'a GPU' if index < 0 else f'cuda:{index}'}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def row_strides(t: torch.Tensor, name: str, index: int) -> Tuple[int, int, int]:
    """Strides of bf16 [rows][tokens][heads][head_dim] with contiguous head rows."""
    stride = t.stride()
    if len(stride) != 4 or t.dtype != torch.bfloat16 or t.get_device() != index or index < 0 \
            or (stride[3] != 1 and t.shape[3] > 1):
        raise ValueError(f"{name} must be bf16 [rows][tokens][heads][head_dim] with contiguous "
                         f"heads on {'a GPU' if index < 0 else f'cuda:{index}'}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    a, b, c, _ = t.shape
    if a == 1 or b == 1 or c == 1:
        # the stride of a dimension of one is never used, and may be anything
        return (stride[0] if a > 1 else 0), (stride[1] if b > 1 else 0), (stride[2] if c > 1 else 0)
    return stride[:3]


def _new_workspace(need: int, device) -> torch.Tensor:
    """Its counters zero; what lies behind them is written before it is read."""
    ws = torch.empty(max(need, _COUNTERS), dtype=torch.uint8, device=device)
    ws[:_COUNTERS].zero_()
    return ws


_COUNTERS = 1 << 18  # bytes that hold every workspace's counters


class Lists:
    """Page lists of (list, key/value head): a table of page numbers with the
    lengths, and for sliding windows the first token that is attended."""

    def __init__(self, pages: torch.Tensor, length: Optional[torch.Tensor], max_len: int,
                 first: Optional[torch.Tensor] = None, extra: int = 0,
                 order: Union[None, bool, Lists] = None):
        """pages: int32 [lists][kv_heads][max_pages], -1 for a dropped page;
        length, first: int32 [lists][kv_heads] or None; max_len: no list is
        longer; extra: added to every length.
        order: in which attention starts the lists.  None sorts them here, longest first
        by `length` and `first` as they are now, which costs 30 to 45 us; False leaves
        them as they are numbered (for lists that are only written and read); another
        Lists gives its own.  An order by other lengths costs time, not results."""
        if pages.dim() != 3:
            raise ValueError("pages must be [lists][kv_heads][max_pages]")
        n, heads, per = pages.shape
        self.index = at = pages.get_device()
        # kept alive with the pointers into them
        self.pages = _device_int32(pages, (n, heads, per), "pages", at)
        self.length = None if length is None else _device_int32(length, (n, heads), "length", at)
        self.first = None if first is None else _device_int32(first, (n, heads), "first", at)
        # longest first: a list that starts late makes the others wait for it (64 x 32
        # lists of 64 to 1024 tokens: 50 us in the order of their numbers, 38 so)
        self.order = None
        if isinstance(order, Lists):
            if (order.n, order.kv_heads, order.index) != (n, heads, at):
                raise ValueError(f"the order of {order.n} x {order.kv_heads} lists on "
                                 f"cuda:{order.index} for {n} x {heads} on cuda:{at}")
            self.order = order.order
        elif order is not None and order is not False:
            raise ValueError("order must be None, False or Lists")
        elif order is None and length is not None and n * heads > 1:
            tokens = length if first is None else length - first
            self.order = torch.argsort(tokens.view(-1), descending=True).to(torch.int32)
        self.arg = B.PagedListsArg(_ptr(pages), _ptr(length), _ptr(first), _ptr(self.order), n, per,
                                   extra, max_len)
        self.n, self.kv_heads = n, heads

    @property
    def extra(self) -> int:
        return self.arg.extra

    def advance(self, tokens: int = 1) -> None:
        """Every list has grown by `tokens` (after a write): counted on the host."""
        self.arg.extra += tokens
        self.arg.max_len += tokens


class PagedKV:
    """A pool of pages and the workspace of its attention.  Use one per stream; a
    graph that has captured its calls counts as work of the stream it is replayed on."""

    def __init__(self, kv_type: str, head_dim: int, kv_heads: int, num_pages: int,
                 page_tokens: int = 64, group: int = 1, device: str = "cuda"):
        """kv_type: "bf16", "int8" or "fp4"; group: query heads per kv head."""
        self.cfg = B.PagedConfig(B.KV_TYPES[kv_type], head_dim, kv_heads, group, page_tokens,
                                 num_pages)
        self.kv_heads, self.head_dim, self.heads = kv_heads, head_dim, kv_heads * group
        self.page_bytes, pool_bytes = B.headkv_paged_plan(self.cfg)
        self.pool = torch.empty(pool_bytes, dtype=torch.uint8, device=device)
        self.device, self.index = self.pool.device, self.pool.get_device()
        self._ws: Optional[torch.Tensor] = None
        self._replaced: List[torch.Tensor] = []  # graphs may hold calls that use them
        self._planned = None

    def lists(self, pages: torch.Tensor, length: Optional[torch.Tensor], max_len: int,
              first: Optional[torch.Tensor] = None, extra: int = 0,
              order: Union[None, bool, Lists] = None) -> Lists:
        got = Lists(pages, length, max_len, first, extra, order)
        self._check_lists(got)
        return got

    def _check_lists(self, lists: Lists) -> None:
        if lists.kv_heads != self.kv_heads:
            raise ValueError(f"lists of {lists.kv_heads} kv heads for a cache of {self.kv_heads}")
        if lists.index != self.index:
            raise ValueError(f"lists on cuda:{lists.index} for a cache on {self.device}")

    def _rows(self, k, v, lists: Lists) -> Tuple[int, Tuple[int, int, int]]:
        shape, ks = k.shape, k.stride()
        if v.stride() != ks or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16 \
                or v.shape != shape or len(shape) != 4 or ks[3] != 1 \
                or k.get_device() != self.index or v.get_device() != self.index:
            ks = self._check_rows(k, v)
        n, tokens, heads, d = shape
        if n != lists.n or heads != self.kv_heads or d != self.head_dim:
            raise ValueError(f"k and v must be [{lists.n}][tokens][{self.kv_heads}]"
                             f"[{self.head_dim}], got {tuple(shape)}")
        if lists.kv_heads != heads or lists.index != self.index:
            self._check_lists(lists)
        if n == 1 or tokens == 1 or heads == 1:
            # the stride of a dimension of one is never used, and may be anything
            return tokens, (ks[0] if n > 1 else 0, ks[1] if tokens > 1 else 0,
                            ks[2] if heads > 1 else 0)
        return tokens, ks[:3]

    def _check_rows(self, k, v):
        for t in (k, v):
            if t.dim() != 4 or t.dtype != torch.bfloat16 or t.shape != k.shape \
                    or t.stride(3) != 1 or t.get_device() != self.index:
                raise ValueError("k and v must be bf16 [lists][tokens][kv_heads][head_dim] with "
                                 f"contiguous rows on {self.device}, got "
                                 f"{t.dtype} {tuple(t.shape)} on {t.device}")
        for i in range(3):
            if k.shape[i] > 1 and k.stride(i) != v.stride(i):
                raise ValueError("k and v must have the same strides")
        return k.stride()

    def write(self, lists: Lists, k: torch.Tensor, v: torch.Tensor,
              counts: Optional[torch.Tensor] = None) -> None:
        """Appends k, v (bf16 [lists][tokens][kv_heads][head_dim], any strides)
        behind the lists' tokens; counts: int32 [lists], tokens of each list."""
        tokens, strides = self._rows(k, v, lists)
        if counts is not None:
            _device_int32(counts, (lists.n,), "counts", self.index)
        B.headkv_paged_write(self.cfg, self.pool.data_ptr(), lists.arg, k.data_ptr(),
                             v.data_ptr(), strides, tokens, _ptr(counts), _stream(self.index))

    def write_rotary(self, lists: Lists, rotary: Rotary, q: Optional[torch.Tensor],
                     k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor],
                     weights: Optional[NormWeights] = None,
                     counts: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """write(), with keys that `rotary` has normalised and turned, and queries: returns
        rotary's of q (bf16 [lists][tokens][heads][head_dim], any strides; None: none).  One
        launch; arguments as for write() and for a call of `rotary`."""
        n, tokens = k.shape[:2]
        if k.shape != (lists.n, tokens, self.kv_heads, self.head_dim) or v.shape != k.shape:
            raise ValueError(f"k and v must be [{lists.n}][tokens][{self.kv_heads}]"
                             f"[{self.head_dim}], got {tuple(k.shape)} and {tuple(v.shape)}")
        if q is not None and q.shape[2:] != (self.heads, self.head_dim):
            raise ValueError(f"q must be [{lists.n}][tokens][{self.heads}][{self.head_dim}], got "
                             f"{tuple(q.shape)}")
        if lists.kv_heads != self.kv_heads or lists.index != self.index:
            self._check_lists(lists)
        call = rotary.rows(q, k, positions, weights, counts, q_out, None, cached=True)
        if call.index != self.index:
            raise ValueError(f"q and k on cuda:{call.index} for a cache on {self.device}")
        B.headkv_paged_write_rotary(self.cfg, self.pool.data_ptr(), lists.arg, rotary.cfg,
                                    rotary._turns, _ptr(positions), tokens, _ptr(counts),
                                    call.q, call.k, v.data_ptr(), row_strides(v, "v", self.index),
                                    _stream(self.index))
        return call.q_out

    def read(self, lists: Lists, tokens: int, begin: int = 0, k: Optional[torch.Tensor] = None,
             v: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Tokens begin .. begin + tokens of every list (begin < 0: counted from
        its end) as bf16 [lists][tokens][kv_heads][head_dim], zeros past the end."""
        if k is None:
            k = torch.empty((lists.n, tokens, self.kv_heads, self.head_dim),
                            dtype=torch.bfloat16, device=self.device)
        if v is None:
            v = torch.empty_like(k)
        got, strides = self._rows(k, v, lists)
        if got != tokens:
            raise ValueError(f"k and v hold {got} tokens, {tokens} are read")
        B.headkv_paged_read(self.cfg, self.pool.data_ptr(), lists.arg, begin, tokens,
                            k.data_ptr(), v.data_ptr(), strides, _stream(self.index))
        return k, v

    def _workspace(self, own: Lists, shared: Optional[Lists],
                   tokens: Optional[int] = None) -> torch.Tensor:
        """Planned once for the lists' tables, for any length that they can hold (fp32
        parts of every query head, of 256 to 1024 own and up to 2048 shared tokens:
        128 rows of 32 query heads of 128 dims with tables of 131072 tokens 270 MB).
        tokens: of attn_tokens(), whose parts are those of as many query heads for each of up
        to 16 columns: as many rows of 16 tokens 550 MB, as a part has up to 8192 tokens from
        4096 lists on, but 127 of them 4.3 GB, of 5 tokens 1.4 GB; with tables of 2^20 tokens
        eight times that.  Tables no longer than the lists get save it."""
        key = (own.pages.shape, None if shared is None else shared.pages.shape, tokens)
        if key == self._planned:
            return self._ws
        most = []
        for l in (own, shared):
            a = None
            if l is not None:
                a = B.PagedListsArg(None, None, None, None, l.arg.lists, l.arg.max_pages, 0,
                                    l.arg.max_pages * self.cfg.page_tokens)
            most.append(a)
        if tokens is None:
            need = B.headkv_paged_attn_plan(self.cfg, *most)
        else:
            need = B.headkv_paged_attn_tokens_plan(self.cfg, *most, tokens)
        if self._ws is None or need > self._ws.numel():
            # twice the last at least: those that are kept take no more than the one in
            # use, however often a table grows
            least = 0 if self._ws is None else 2 * self._ws.numel()
            ws = _new_workspace(max(need, least), self.device)
            if torch.cuda.is_current_stream_capturing():
                return ws  # the graph's memory, zeroed by it: for this call only
            if self._ws is not None:
                self._replaced.append(self._ws)
            self._ws = ws
        self._planned = key
        return self._ws

    def attn(self, own: Lists, q: torch.Tensor, shared: Optional[Lists] = None,
             share: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q (bf16 [batch][kv_heads * group][head_dim], rows of any
        stride) over the rows' own lists and the shared ones that `share` (int32
        [batch], list number or -1) names; fp32 out, and lse if given."""
        batch, heads, d = own.n, self.heads, self.head_dim
        if q.dtype != torch.bfloat16 or q.shape != (batch, heads, d) \
                or q.get_device() != self.index:
            raise ValueError(f"q must be bf16 {(batch, heads, d)} on {self.device}")
        row, step, one = q.stride()
        if one != 1 or (step != d and heads > 1):
            raise ValueError("q must have contiguous rows")
        if out is None:
            out = torch.empty((batch, heads, d), dtype=torch.float32, device=self.device)
        elif out.dtype != torch.float32 or out.shape != (batch, heads, d) \
                or out.get_device() != self.index or not out.is_contiguous():
            raise ValueError(f"out must be contiguous float32 {(batch, heads, d)} on {self.device}")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (batch, heads)
                                or lse.get_device() != self.index or not lse.is_contiguous()):
            raise ValueError(f"lse must be contiguous float32 {(batch, heads)} on {self.device}")
        for l in (own,) if shared is None else (own, shared):
            if l.kv_heads != self.kv_heads or l.index != self.index:
                self._check_lists(l)
        if share is not None:
            _device_int32(share, (batch,), "share", self.index)
        stream = _stream(self.index)
        ws = self._workspace(own, shared)
        B.headkv_paged_attn(self.cfg, self.pool.data_ptr(), own.arg,
                            None if shared is None else shared.arg, _ptr(share), q.data_ptr(),
                            row if batch > 1 else 0, out.data_ptr(), _ptr(lse), ws.data_ptr(),
                            ws.numel(), stream)
        return out

    def attn_tokens(self, own: Lists, q: torch.Tensor, counts: Optional[torch.Tensor] = None,
                    window: Optional[torch.Tensor] = None, shared: Optional[Lists] = None,
                    share: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q (bf16 [batch][tokens][kv_heads * group][head_dim], any strides of
        rows and tokens), tokens that have been written behind the rows' own lists: each
        attends what is before it, itself, and with window (int32 [batch][kv_heads], 0: none)
        so many tokens of its list at most.  counts: int32 [batch], tokens of each row, behind
        which results are left as they are.  shared, share, out, lse: as for attn()."""
        if q.dim() != 4 or q.dtype != torch.bfloat16 or q.get_device() != self.index \
                or q.shape[0] != own.n or q.shape[2:] != (self.heads, self.head_dim):
            raise ValueError(f"q must be bf16 [{own.n}][tokens][{self.heads}][{self.head_dim}] "
                             f"on {self.device}, got {q.dtype} {tuple(q.shape)} on {q.device}")
        batch, tokens, heads, d = q.shape
        row, token, step, one = q.stride()
        if tokens and (one != 1 or (step != d and heads > 1)):
            raise ValueError("the heads of a token of q must be contiguous")
        if out is None:
            # what counts leave out is left as it is: zeros in what is allocated here
            empty = torch.empty if counts is None else torch.zeros
            out = empty(q.shape, dtype=torch.float32, device=self.device)
        elif out.dtype != torch.float32 or out.shape != q.shape \
                or out.get_device() != self.index or not out.is_contiguous():
            raise ValueError(f"out must be contiguous float32 {tuple(q.shape)} on {self.device}")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:3]
                                or lse.get_device() != self.index or not lse.is_contiguous()):
            raise ValueError(f"lse must be contiguous float32 {tuple(q.shape[:3])} on "
                             f"{self.device}")
        for l in (own,) if shared is None else (own, shared):
            if l.kv_heads != self.kv_heads or l.index != self.index:
                self._check_lists(l)
        if share is not None:
            _device_int32(share, (batch,), "share", self.index)
        if counts is not None:
            _device_int32(counts, (batch,), "counts", self.index)
        if window is not None:
            _device_int32(window, (batch, self.kv_heads), "window", self.index)
        stream = _stream(self.index)
        ws = self._workspace(own, shared, tokens)
        B.headkv_paged_attn_tokens(self.cfg, self.pool.data_ptr(), own.arg,
                                   None if shared is None else shared.arg, _ptr(share), tokens,
                                   _ptr(counts), _ptr(window), q.data_ptr(),
                                   (row if batch > 1 else 0, token if tokens > 1 else 0),
                                   out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(), stream)
        return out


_LOGITS = {torch.bfloat16: B.HEADKV_LOGITS_BF16, torch.float32: B.HEADKV_LOGITS_F32}
_score_ws: Dict[Tuple[int, int], torch.Tensor] = {}  # per device and stream


_score_need = lru_cache(256)(B.headkv_logprobs_plan)  # bytes of workspace


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0,
                   temperature: float = 1.0) -> Dict[str, torch.Tensor]:
    """Scores of `tokens` (int32 [rows]) under softmax(logits / temperature),
    logits [rows][vocab] bf16 or float32 with rows of any stride: "logprob",
    "entropy" and "rank" per row, and with top > 0 "top_logprob" and "top_index"
    [rows][top]."""
    if top < 0:
        raise ValueError("top must be >= 0")
    index = logits.get_device()
    if logits.dim() != 2 or logits.dtype not in _LOGITS or logits.stride(1) != 1 or index < 0:
        raise ValueError("logits must be bf16 or float32 [rows][vocab] with contiguous rows on "
                         "the GPU")
    rows, vocab = logits.shape
    _device_int32(tokens, (rows,), "tokens", index)
    stream = _stream(index)
    dev = logits.device
    # one allocation for all results: an empty tensor costs 1.3 us of the 4 that the
    # call itself takes, a view of one 0.4
    many = rows * top
    buf = torch.empty(3 * rows + 2 * many, dtype=torch.float32, device=dev)
    if top > 0:
        logprob, entropy, rank, best, which = buf.split_with_sizes((rows, rows, rows, many, many))
        res = {"logprob": logprob, "entropy": entropy, "rank": rank.view(torch.int32),
               "top_logprob": best.view(rows, top),
               "top_index": which.view(torch.int32).view(rows, top)}
    else:
        logprob, entropy, rank = buf.split_with_sizes((rows, rows, rows))
        res = {"logprob": logprob, "entropy": entropy, "rank": rank.view(torch.int32)}
    need = _score_need(rows, vocab, top)
    ws = None
    if need:
        if torch.cuda.is_current_stream_capturing():
            # the graph's memory, zeroed by it: graphs may be replayed on other streams
            ws = _new_workspace(need, dev)
        else:
            key = (index, stream)
            ws = _score_ws.get(key)
            if ws is None or ws.numel() < need:
                ws = _score_ws[key] = _new_workspace(need, dev)
    B.headkv_token_logprobs(logits.data_ptr(), _LOGITS[logits.dtype], rows, vocab,
                            logits.stride(0) if rows > 1 else vocab, tokens.data_ptr(),
                            temperature, top, logprob.data_ptr(), entropy.data_ptr(),
                            rank.data_ptr(), best.data_ptr() if top > 0 else None,
                            which.data_ptr() if top > 0 else None, _ptr(ws),
                            0 if ws is None else ws.numel(), stream)
    return res
