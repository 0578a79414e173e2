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
from .paged import _device_int32, _stream, row_strides
from .session import _ptr


class _Pair:
    """A weight and a bias, checked once."""
    __slots__ = ("weight", "bias", "arg", "heads", "dim", "index")

    def __init__(self, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], name: str):
        self.weight, self.bias = weight, bias  # kept alive with the pointers into them
        self.heads = self.dim = self.index = None
        for w in (weight, bias):
            if w is None:
                continue
            if w.dtype != torch.float32 or w.dim() not in (1, 2) or w.get_device() < 0 \
                    or not w.is_contiguous():
                raise ValueError(f"{name}'s weights must be contiguous float32 [head_dim] or "
                                 f"[heads][head_dim] on the GPU, got {w.dtype} {tuple(w.shape)} "
                                 f"on {w.device}")
            self.heads = w.shape[0] if w.dim() == 2 else None
            self.dim, self.index = w.shape[-1], w.get_device()
        if weight is not None and bias is not None \
                and (weight.shape != bias.shape or weight.device != bias.device):
            raise ValueError(f"{name}'s weight and bias must have one shape and device")
        self.arg = _ptr(weight), _ptr(bias), int(self.heads is not None)


class NormWeights:
    """Weights and biases of the norms: float32 [head_dim] for all heads or [heads][head_dim]
    for each (both of a pair the same), contiguous; None: ones and zeros."""

    def __init__(self, q_weight: Optional[torch.Tensor] = None,
                 q_bias: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 k_bias: Optional[torch.Tensor] = None):
        self.q, self.k = _Pair(q_weight, q_bias, "q"), _Pair(k_weight, k_bias, "k")


_ONES = NormWeights()


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
        self._turns = _ptr(self.turns)

    def _arg(self, t, out, pair, name) -> B.RotaryRowsArg:
        index, shape = self.index, t.shape
        strides = row_strides(t, name, index)
        if shape[3] != self.head_dim:
            raise ValueError(f"{name} has heads of {shape[3]} dims, not {self.head_dim}")
        to, at = (0, 0, 0), None
        if out is not None:
            if out.shape != shape:
                raise ValueError(f"{name}_out must be {tuple(shape)}, got {tuple(out.shape)}")
            to, at = row_strides(out, name + "_out", index), out.data_ptr()
        heads, w = shape[2], (None, None, 0)
        if self.normed and pair.dim is not None:
            if pair.dim != self.head_dim or pair.index != index \
                    or (pair.heads is not None and pair.heads != heads):
                raise ValueError(f"{name}'s weights must be [{self.head_dim}] or [{heads}]"
                                 f"[{self.head_dim}] on cuda:{index}, got [{pair.heads}]"
                                 f"[{pair.dim}] on cuda:{pair.index}")
            w = pair.arg
        return B.RotaryRowsArg(t.data_ptr(), at, *strides, *to, w[0], w[1], heads, w[2])

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
        w = weights or _ONES
        # what counts leave out is left as it is: zeros in what is allocated here
        empty = torch.empty if counts is None else torch.zeros
        if q is not None and q_out is None:
            q_out = empty(q.shape, dtype=torch.bfloat16, device=q.device)
        if k is not None and k_out is None and not cached:
            k_out = empty(k.shape, dtype=torch.bfloat16, device=k.device)
        return _Call(None if q is None else self._arg(q, q_out, w.q, "q"),
                     None if k is None else self._arg(k, k_out, w.k, "k"),
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
        B.headkv_rotary(self.cfg, self._turns, _ptr(positions), call.rows, call.tokens,
                        _ptr(counts), call.q, call.k, _stream(self.index))
        return call.q_out, call.k_out
