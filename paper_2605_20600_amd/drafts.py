"""Verification of drafted tokens against the target's probabilities, from given random
numbers: what a row keeps is distributed as if the target had sampled it.

PyTorch supplies device memory and the stream, as for Session; the computation is a
call into libheadkv.so through the binding.  Calls are made on the current device and
its current stream; tensors that lie elsewhere are refused.
"""
from __future__ import annotations

from functools import lru_cache
from typing import Dict, Optional, Tuple

import torch

from . import binding as B
from .paged import _LOGITS, _device_int32, _new_workspace, _stream
from .session import _ptr

_verify_ws: Dict[Tuple[int, int], torch.Tensor] = {}  # per device and stream


_verify_need = lru_cache(256)(B.headkv_verify_plan)  # bytes of workspace


def _logit_strides(t: torch.Tensor, shape: Tuple[int, int, int], dtype, index: int,
                   name: str) -> Tuple[int, int]:
    if t.dtype != dtype or t.shape != shape or t.get_device() != index \
            or (shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be {dtype} {shape} on cuda:{index} with contiguous rows, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    # the stride of a dimension of one is never used, and may be anything
    return (t.stride(0) if shape[0] > 1 else 0), (t.stride(1) if shape[1] > 1 else 0)


def verify_drafts(logits: torch.Tensor, tokens: torch.Tensor, uniforms: torch.Tensor,
                  draft_logits: Optional[torch.Tensor] = None,
                  counts: Optional[torch.Tensor] = None,
                  temperature: float = 1.0) -> Dict[str, torch.Tensor]:
    """Drafts `tokens` (int32 [rows][drafts]) against logits ([rows][drafts + 1][vocab], bf16
    or float32, rows of any strides).  draft_logits ([rows][drafts][vocab], of the same type)
    are what they were sampled from, None: each was certain; uniforms: float32 [rows][drafts
    + 1], the last one for the next token; counts: int32 [rows], drafts of each row, negative
    for a row that is left out; temperature 0 takes the largest logits.
    Returns "tokens" [rows][drafts + 1], what each row gains, -1 behind it, "count" [rows],
    how many that are, and "logprob" [rows][drafts + 1], 0 behind them."""
    index = logits.get_device()
    if logits.dim() != 3 or logits.dtype not in _LOGITS or index < 0 or logits.shape[1] < 1:
        raise ValueError("logits must be bf16 or float32 [rows][drafts + 1][vocab] on the GPU")
    rows, places, vocab = logits.shape
    drafts = places - 1
    strides = _logit_strides(logits, (rows, places, vocab), logits.dtype, index, "logits")
    more = (0, 0)
    if draft_logits is not None:
        more = _logit_strides(draft_logits, (rows, drafts, vocab), logits.dtype, index,
                              "draft_logits")
    _device_int32(tokens, (rows, drafts), "tokens", index)
    if counts is not None:
        _device_int32(counts, (rows,), "counts", index)
    if uniforms.dtype != torch.float32 or uniforms.shape != (rows, places) \
            or uniforms.get_device() != index or not uniforms.is_contiguous():
        raise ValueError(f"uniforms must be contiguous float32 {(rows, places)} on cuda:{index}")
    stream = _stream(index)
    dev = logits.device
    # one allocation for all results
    n = rows * places
    buf = torch.empty(2 * n + rows, dtype=torch.int32, device=dev)
    kept, logprob, count = buf.split_with_sizes((n, n, rows))
    need = _verify_need(rows, drafts, vocab)
    if torch.cuda.is_current_stream_capturing():
        # the graph's memory, zeroed by it: graphs may be replayed on other streams
        ws = _new_workspace(need, dev)
    else:
        key = (index, stream)
        ws = _verify_ws.get(key)
        if ws is None or ws.numel() < need:
            ws = _verify_ws[key] = _new_workspace(need, dev)
    B.headkv_verify_drafts(logits.data_ptr(), _ptr(draft_logits), _LOGITS[logits.dtype], rows,
                           drafts, vocab, (*strides, *more), _ptr(tokens), _ptr(counts),
                           uniforms.data_ptr(), temperature, kept.data_ptr(), count.data_ptr(),
                           logprob.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    return {"tokens": kept.view(rows, places), "count": count,
            "logprob": logprob.view(torch.float32).view(rows, places)}
