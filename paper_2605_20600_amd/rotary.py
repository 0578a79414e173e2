"""Norms of queries and keys with rotary positions, for keys that are cached as they
are attended.

PyTorch supplies device memory and the stream, as for Session; every computation is a
call into libheadkv.so through the binding.  Calls are made on the current device and
its current stream; tensors that lie elsewhere are refused.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B
from .session import _ptr


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
    if t.dim() != 4 or t.dtype != torch.bfloat16 or t.get_device() != index or index < 0 \
            or (t.stride(3) != 1 and t.shape[3] > 1):
        raise ValueError(f"{name} must be bf16 [rows][tokens][heads][head_dim] with contiguous "
                         f"heads on {'a GPU' if index < 0 else f'cuda:{index}'}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    # the stride of a dimension of one is never used, and may be anything
    a, b, c = (s if n > 1 else 0 for s, n in zip(t.stride()[:3], t.shape))
    return a, b, c


class NormWeights(NamedTuple):
    """Weights and biases of the norms: float32 [head_dim] for all heads or [heads][head_dim]
    for each (both of a pair the same), contiguous; None: ones and zeros."""
    q_weight: Optional[torch.Tensor] = None
    q_bias: Optional[torch.Tensor] = None
    k_weight: Optional[torch.Tensor] = None
    k_bias: Optional[torch.Tensor] = None


class _Call(NamedTuple):
    q: Optional[B.RotaryRowsArg]
    k: Optional[B.RotaryRowsArg]
    q_out: Optional[torch.Tensor]
    k_out: Optional[torch.Tensor]
    index: int
    rows: int
    tokens: int


class Rotary:
    """A rotation, with the norm before it; its table of angles lies on `device`."""

    def __init__(self, head_dim: int, rotary_dims: Optional[int] = None, layout: str = "half",
                 axes: int = 1, norm: Optional[str] = None, eps: float = 1e-6,
                 base: float = 10000.0, scaling: Optional[tuple] = None, scale: float = 1.0,
                 device: str = "cuda"):
        """rotary_dims: of a head, its first ones (None: all); layout: "half" or "pairs";
        axes: coordinates of a position; norm: None, "rms" or "layer"; scaling: None,
        ("linear", factor), ("base", factor) or ("bands", factor, original length, low,
        high); scale: of what is turned."""
        if layout not in B.ROPE_LAYOUTS or norm not in B.NORMS:
            raise ValueError(f"unknown layout {layout!r} or norm {norm!r}")
        kind = "none" if scaling is None else scaling[0]
        kinds = {"none": (B.HEADKV_SCALE_NONE, 1), "linear": (B.HEADKV_SCALE_LINEAR, 2),
                 "base": (B.HEADKV_SCALE_BASE, 2), "bands": (B.HEADKV_SCALE_BANDS, 5)}
        if kind not in kinds or (scaling is not None and len(scaling) != kinds[kind][1]):
            raise ValueError(f"unknown scaling {scaling!r}")
        factor, original, low, high = (tuple(scaling or ())[1:] + (0.0,) * 4)[:4]
        self.cfg = B.RotaryConfig(head_dim, head_dim if rotary_dims is None else rotary_dims,
                                  B.ROPE_LAYOUTS[layout], axes, B.NORMS[norm], eps, scale,
                                  kinds[kind][0], int(original), base, factor, low, high)
        self.head_dim, self.axes, self.normed = head_dim, axes, norm is not None
        self.turns = torch.tensor(B.headkv_rotary_plan(self.cfg), dtype=torch.float64,
                                  device=device)
        self.index = self.turns.get_device()

    def _arg(self, t, out, weight, bias, name) -> B.RotaryRowsArg:
        strides = row_strides(t, name, self.index)
        if t.shape[3] != self.head_dim:
            raise ValueError(f"{name} has heads of {t.shape[3]} dims, not {self.head_dim}")
        to = (0, 0, 0)
        if out is not None:
            if out.shape != t.shape:
                raise ValueError(f"{name}_out must be {tuple(t.shape)}, got {tuple(out.shape)}")
            to = row_strides(out, name + "_out", self.index)
        heads = t.shape[2]
        per_head = 0
        if self.normed:
            for w in (weight, bias):
                if w is None:
                    continue
                if w.dtype != torch.float32 or w.get_device() != self.index \
                        or not w.is_contiguous() \
                        or w.shape not in ((self.head_dim,), (heads, self.head_dim)):
                    raise ValueError(f"{name}'s weights must be contiguous float32 [head_dim] or "
                                     f"[{heads}][head_dim] on cuda:{self.index}, got {w.dtype} "
                                     f"{tuple(w.shape)} on {w.device}")
                per_head = w.dim() - 1
            if weight is not None and bias is not None and weight.shape != bias.shape:
                raise ValueError(f"{name}'s weight and bias must have one shape")
        return B.RotaryRowsArg(t.data_ptr(), _ptr(out), *strides, *to,
                               _ptr(weight) if self.normed else None,
                               _ptr(bias) if self.normed else None, heads, per_head)

    def rows(self, q, k, positions, weights, counts, q_out, k_out, cached=False) -> _Call:
        """The checked arguments of a call; cached: the keys' results go to a cache."""
        some = k if k is not None else q
        if some is None:
            raise ValueError("q and k are both None")
        if some.dim() != 4 or (q is not None and q.shape[:2] != some.shape[:2]):
            raise ValueError("q and k must be [rows][tokens][heads][head_dim] of the same rows "
                             "and tokens")
        rows, tokens = some.shape[:2]
        if self.cfg.rotary_dims:
            if positions is None:
                raise ValueError("positions are needed")
            shape = (rows, tokens, self.axes)
            if positions.dim() == 2 and self.axes == 1:
                shape = shape[:2]
            _device_int32(positions, shape, "positions", self.index)
        if counts is not None:
            _device_int32(counts, (rows,), "counts", self.index)
        w = weights or NormWeights()
        # what counts leave out is left as it is: zeros in what is allocated here
        empty = torch.empty if counts is None else torch.zeros
        if q is not None and q_out is None:
            q_out = empty(q.shape, dtype=torch.bfloat16, device=q.device)
        if k is not None and k_out is None and not cached:
            k_out = empty(k.shape, dtype=torch.bfloat16, device=k.device)
        return _Call(None if q is None else self._arg(q, q_out, w.q_weight, w.q_bias, "q"),
                     None if k is None else self._arg(k, k_out, w.k_weight, w.k_bias, "k"),
                     q_out, k_out, self.index, rows, tokens)

    def __call__(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                 positions: Optional[torch.Tensor], weights: Optional[NormWeights] = None,
                 counts: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None
                 ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        """q, k (bf16 [rows][tokens][heads][head_dim], heads' rows contiguous, any other
        strides; either may be None) normalised and turned to `positions` (int32
        [rows][tokens][axes], with one axis also [rows][tokens]).  counts (int32 [rows]):
        tokens of each row, behind which results are left as they are.  q_out and k_out may
        be q and k themselves."""
        call = self.rows(q, k, positions, weights, counts, q_out, k_out)
        B.headkv_rotary(self.cfg, _ptr(self.turns), _ptr(positions), call.rows, call.tokens,
                        _ptr(counts), call.q, call.k, _stream(self.index))
        return call.q_out, call.k_out
