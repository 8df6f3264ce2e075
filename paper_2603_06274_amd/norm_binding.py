"""ctypes binding of the entry points in include/stem_norm.h: heads normalised, weighted and turned by their positions in one pass.

Function names and argument order follow the header; shapes and pages are decode_binding's.  A call checks that the tensors it gets are
of the shape's types and sizes and on the current device, and passes their addresses.  Every step runs inside the library's HIP
kernels on torch's current stream; there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .decode_binding import (DTYPES, PageShape, RotaryShape, _check, _f32, _here, _i32, _need, _sz, _values, _vp, _whole, lib as _decode_lib,
                             stem_pages, stem_rotary_shape)

EXPORTED = ["stem_norm_rotary", "stem_norm_rotary_append", "stem_norm_rotary_backward_workspace_bytes", "stem_norm_rotary_backward"]


class stem_head_norm(ctypes.Structure):
    _fields_ = [("q_weight", _vp), ("k_weight", _vp), ("weight_dtype", _i32), ("weight_offset", _f32), ("eps", _f32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The library that binding.lib() loads, with these entry points' signatures.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _decode_lib()
        rot, norm, pages = (ctypes.POINTER(x) for x in (stem_rotary_shape, stem_head_norm, stem_pages))
        sigs = {
            "stem_norm_rotary": [rot, norm, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _vp],
            "stem_norm_rotary_append": [rot, norm, pages, _vp, _vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _vp],
            "stem_norm_rotary_backward_workspace_bytes": [rot, ctypes.POINTER(_sz)],
            "stem_norm_rotary_backward": [rot, norm, _vp, _vp, _vp, _vp, _f32] + [_vp] * 7 + [_sz, _vp],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = L
    return _lib


class HeadNorm:
    """The norm of the heads of queries and keys: weights [head_dim] of one type (either may be None: no weights), to which weight_offset is
    added.  The tensors are used where they are at every call, so weights that are updated in place count as they are then."""

    def __init__(self, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], eps: float = 1e-6, weight_offset: float = 0.0):
        given = [w for w in (q_weight, k_weight) if w is not None]
        for w in given:
            _need(w.dim() == 1 and w.is_contiguous() and w.dtype in DTYPES, "weights have to be contiguous [head_dim] of a supported type")
            _need(w.dtype is given[0].dtype and w.shape == given[0].shape and w.device == given[0].device, "weights have to be alike")
        self.q_weight, self.k_weight, self.eps, self.weight_offset = q_weight, k_weight, float(eps), float(weight_offset)
        _need(math.isfinite(self.weight_offset) and 2.0 ** -126 <= _f32(self.eps).value < math.inf, "eps or weight_offset cannot be used")
        self.head_dim = given[0].numel() if given else None
        self.dtype = DTYPES[given[0].dtype] if given else 0

    def need_fits(self, head_dim: int, device: torch.device) -> None:
        """Raises unless heads of head_dim values on `device` can be normalised by it."""
        for w in (self.q_weight, self.k_weight):
            if w is not None:
                _need(w.numel() == head_dim and w.device == device and not w.data_ptr() & 15,
                      "weights have to be of %d values at whole 16 bytes, on the heads' device" % head_dim)

    def at(self, head_dim: int, dev: int):
        """The structure for a call."""
        if self.head_dim not in (None, head_dim):
            raise ValueError("weights of %d values for heads of %d" % (self.head_dim, head_dim))
        return ctypes.byref(stem_head_norm(self._address(self.q_weight, dev), self._address(self.k_weight, dev), self.dtype,
                                           self.weight_offset, self.eps))

    @staticmethod
    def _address(w: Optional[torch.Tensor], dev: int) -> Optional[int]:
        if w is None:
            return None
        if w.get_device() != dev:
            raise ValueError("weights have to be on the current device")
        return w.data_ptr()


def stem_norm_rotary(shape: RotaryShape, norm: HeadNorm, q, k, positions: torch.Tensor, turns: torch.Tensor, attention_factor: float, q_out,
                     k_out) -> None:
    dev, stream = _here()
    _check(lib().stem_norm_rotary(shape.ref, norm.at(shape.c.head_dim, dev), _values(q, shape.q, "q", dev), _values(k, shape.k, "k", dev),
                                  _whole(positions, shape.tokens, "positions", dev),
                                  _whole(turns, shape.pairs, "turns", dev, torch.float64), attention_factor,
                                  _values(q_out, shape.q_out, "q_out", dev), _values(k_out, shape.k_out, "k_out", dev), stream),
           "stem_norm_rotary")


def stem_norm_rotary_append(shape: RotaryShape, norm: HeadNorm, pages: PageShape, q, k, v, positions: torch.Tensor, slots: torch.Tensor,
                            turns: torch.Tensor, attention_factor: float, q_out, k_pages: torch.Tensor, v_pages: torch.Tensor) -> None:
    dev, stream = _here()
    _need(pages.heads == shape.c.num_kv_heads and pages.head_dim == shape.c.head_dim and
          (shape.k is None or pages.seen[2] == shape.k[2]), "the pages do not go with k")
    _check(lib().stem_norm_rotary_append(
        shape.ref, norm.at(shape.c.head_dim, dev), pages.ref, _values(q, shape.q, "q", dev), _values(k, shape.k, "k", dev),
        _values(v, shape.k, "v", dev), _whole(positions, shape.tokens, "positions", dev), _whole(slots, shape.tokens, "slots", dev),
        _whole(turns, shape.pairs, "turns", dev, torch.float64), attention_factor, _values(q_out, shape.q_out, "q_out", dev),
        _values(k_pages, pages.seen, "k_pages", dev), _values(v_pages, pages.seen, "v_pages", dev), stream), "stem_norm_rotary_append")


def stem_norm_rotary_backward_workspace_bytes(shape: RotaryShape) -> int:
    n = _sz()
    _check(lib().stem_norm_rotary_backward_workspace_bytes(shape.ref, ctypes.byref(n)), "stem_norm_rotary_backward_workspace_bytes")
    return n.value


def stem_norm_rotary_backward(shape: RotaryShape, norm: HeadNorm, q, k, positions: torch.Tensor, turns: torch.Tensor,
                              attention_factor: float, grad_q, grad_k, q_grad, k_grad, q_weight_grad: Optional[torch.Tensor],
                              k_weight_grad: Optional[torch.Tensor], workspace: Optional[torch.Tensor]) -> None:
    """grad_q and grad_k are as the shape's q_out and k_out, q_grad and k_grad as its q and k."""
    dev, stream = _here()
    d = shape.c.head_dim
    _check(lib().stem_norm_rotary_backward(
        shape.ref, norm.at(d, dev), _values(q, shape.q, "q", dev), _values(k, shape.k, "k", dev),
        _whole(positions, shape.tokens, "positions", dev), _whole(turns, shape.pairs, "turns", dev, torch.float64), attention_factor,
        _values(grad_q, shape.q_out, "grad_q", dev), _values(grad_k, shape.k_out, "grad_k", dev),
        _values(q_grad, shape.q, "q_grad", dev), _values(k_grad, shape.k, "k_grad", dev),
        None if q_weight_grad is None else _whole(q_weight_grad, d, "q_weight_grad", dev, torch.float32),
        None if k_weight_grad is None else _whole(k_weight_grad, d, "k_weight_grad", dev, torch.float32),
        None if workspace is None else _whole(workspace, 0, "workspace", dev, torch.uint8),
        0 if workspace is None else workspace.numel(), stream), "stem_norm_rotary_backward")
