"""ctypes binding of the entry points in include/stem_tree.h: trees of drafted tokens, their attention, and what is kept of them.

Function names and argument order follow the header; pages and the attention's shape are decode_binding's.  A call checks that the tensors
it gets are of the shape's types and sizes and on the current device, and passes their addresses.  Every step runs inside the
library's HIP kernels on torch's current stream; there is no fallback.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .decode_binding import (DTYPES, STEM_MAX_HEAD_DIM, PageShape, PrefixShape, _check, _f32, _here, _i32, _lines, _need, _sz, _values, _vp, _whole,
                             lib as _decode_lib, stem_pages, stem_prefix_shape)

STEM_MAX_TREE = 1024

EXPORTED = ["stem_tree_masks", "stem_tree_attn_workspace_bytes", "stem_tree_attn", "stem_tree_accept_workspace_bytes", "stem_tree_accept",
            "stem_tree_commit"]


class stem_tree_shape(ctypes.Structure):
    _fields_ = [(x, _i32) for x in ("requests", "tokens", "max_new", "position_offset")]


class stem_accept_shape(ctypes.Structure):
    _fields_ = [(x, _i32) for x in ("requests", "tokens", "max_new", "page_size", "num_pages", "pages_per_request", "id_bits")]


_lib = None


def lib() -> ctypes.CDLL:
    """The library that binding.lib() loads, with these entry points' signatures.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _decode_lib()
        tree, pre, acc, pages, size = (ctypes.POINTER(x) for x in (stem_tree_shape, stem_prefix_shape, stem_accept_shape, stem_pages, _sz))
        sigs = {
            "stem_tree_masks": [tree] + [_vp] * 7,
            "stem_tree_attn_workspace_bytes": [pre, size],
            "stem_tree_attn": [pre] + [_vp] * 9 + [_f32, _vp, _vp, _vp, _sz, _vp],
            "stem_tree_accept_workspace_bytes": [acc, size],
            "stem_tree_accept": [acc] + [_vp] * 15 + [_sz, _vp],
            "stem_tree_commit": [acc, pages, _i32, _i32, _i32] + [_vp] * 6,
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = L
    return _lib


def mask_words(max_new: int) -> int:
    """64-bit words of a token's mask."""
    return (int(max_new) + 63) // 64


class TreeShape:
    """Sizes of a step whose new tokens form trees."""

    def __init__(self, requests: int, tokens: int, max_new: int, position_offset: int = 0):
        self.c = stem_tree_shape(int(requests), int(tokens), int(max_new), int(position_offset))
        self.sizes = int(requests), int(tokens), mask_words(max_new)
        self.ref = ctypes.byref(self.c)


def stem_tree_masks(shape: TreeShape, parents: torch.Tensor, lens: torch.Tensor, cu_new: torch.Tensor, positions: Optional[torch.Tensor],
                    masks: torch.Tensor, status: torch.Tensor) -> None:
    dev, stream = _here()
    R, T, W = shape.sizes
    _check(lib().stem_tree_masks(shape.ref, _whole(parents, T, "parents", dev), _whole(lens, R, "lens", dev),
                                 _whole(cu_new, R + 1, "cu_new", dev), None if positions is None else _whole(positions, T, "positions", dev),
                                 _lines(masks, T, W, "masks", dev, torch.int64), _whole(status, 1, "status", dev), stream),
           "stem_tree_masks")


def stem_tree_attn_workspace_bytes(shape: PrefixShape) -> int:
    n = _sz()
    _check(lib().stem_tree_attn_workspace_bytes(shape.ref, ctypes.byref(n)), "stem_tree_attn_workspace_bytes")
    return n.value


def stem_tree_attn(shape: PrefixShape, q: torch.Tensor, prefix_k, prefix_v, k_pages, v_pages, table, lens, cu_new: torch.Tensor,
                   masks: torch.Tensor, softmax_scale: float, out: torch.Tensor, lse: Optional[torch.Tensor],
                   workspace: torch.Tensor) -> None:
    dev, stream = _here()
    R, W, paged, Hq, T = shape.sizes
    _check(lib().stem_tree_attn(
        shape.ref, _values(q, shape.q, "q", dev), _values(prefix_k, shape.prefix, "prefix_k", dev),
        _values(prefix_v, shape.prefix, "prefix_v", dev), _values(k_pages, shape.pages, "k_pages", dev) if paged else None,
        _values(v_pages, shape.pages, "v_pages", dev) if paged else None,
        _lines(table, R, W, "table", dev) if paged else None, _whole(lens, R, "lens", dev) if paged else None,
        _whole(cu_new, R + 1, "cu_new", dev), _lines(masks, T, mask_words(shape.c.max_new), "masks", dev, torch.int64), softmax_scale,
        _values(out, shape.q, "out", dev), None if lse is None else _lines(lse, Hq, T, "lse", dev, torch.float32),
        _whole(workspace, 0, "workspace", dev, torch.uint8), workspace.numel(), stream), "stem_tree_attn")


class AcceptShape:
    """Sizes of a step of which some tokens are kept."""

    def __init__(self, requests: int, tokens: int, max_new: int, page_size: int, num_pages: int, pages_per_request: int):
        self.c = {t: stem_accept_shape(int(requests), int(tokens), int(max_new), int(page_size), int(num_pages), int(pages_per_request), bits)
                  for t, bits in ((torch.int32, 32), (torch.int64, 64))}
        self.sizes = int(requests), int(tokens), int(num_pages), int(pages_per_request)     # what its tensors go by
        self.ref = {t: ctypes.byref(c) for t, c in self.c.items()}


def stem_tree_accept_workspace_bytes(shape: AcceptShape) -> int:
    n = _sz()
    _check(lib().stem_tree_accept_workspace_bytes(shape.ref[torch.int64], ctypes.byref(n)), "stem_tree_accept_workspace_bytes")
    return n.value


def stem_tree_accept(shape: AcceptShape, parents: torch.Tensor, draft_ids: torch.Tensor, target_ids: torch.Tensor, cu_new: torch.Tensor,
                     lens: torch.Tensor, ring_state: torch.Tensor, ring: torch.Tensor, table: torch.Tensor, lens_out: torch.Tensor,
                     ring_state_out: torch.Tensor, accepted: torch.Tensor, path: torch.Tensor, next_ids: torch.Tensor, status: torch.Tensor,
                     workspace: torch.Tensor) -> None:
    """draft_ids, target_ids and next_ids are int32 or int64, all three."""
    dev, stream = _here()
    R, T, N, W = shape.sizes
    ids = draft_ids.dtype
    _need(ids in shape.ref, "draft_ids: %s is not supported" % ids)
    _check(lib().stem_tree_accept(
        shape.ref[ids], _whole(parents, T, "parents", dev), _whole(draft_ids, T, "draft_ids", dev, ids),
        _whole(target_ids, T, "target_ids", dev, ids), _whole(cu_new, R + 1, "cu_new", dev), _whole(lens, R, "lens", dev),
        _whole(ring_state, 2, "ring_state", dev), _whole(ring, N, "ring", dev), _lines(table, R, W, "table", dev),
        _whole(lens_out, R, "lens_out", dev), _whole(ring_state_out, 2, "ring_state_out", dev), _whole(accepted, R, "accepted", dev),
        _whole(path, T, "path", dev), _whole(next_ids, R, "next_ids", dev, ids), _whole(status, 2, "status", dev),
        _whole(workspace, 0, "workspace", dev, torch.uint8), workspace.numel(), stream), "stem_tree_accept")


def need_movable_rows(pages: PageShape) -> None:
    """What stem_tree_commit asks of pages beyond what their block table does: types and sizes of rows."""
    d, dtype = pages.head_dim, pages.seen[2]
    if dtype not in DTYPES or d % 8 or d > STEM_MAX_HEAD_DIM or pages.heads < 1 or pages.heads * d * dtype.itemsize > 1 << 26:
        raise ValueError("rows of %d heads of %d values of %s cannot be moved" % (pages.heads, d, dtype))


def stem_tree_commit(shape: AcceptShape, pages: PageShape, path: torch.Tensor, slots: torch.Tensor, cu_new: torch.Tensor,
                     k_pages: torch.Tensor, v_pages: torch.Tensor) -> None:
    dev, stream = _here()
    R, T = shape.sizes[:2]
    dtype = pages.seen[2]
    _need(dtype in DTYPES, "pages: %s is not supported" % dtype)
    _check(lib().stem_tree_commit(shape.ref[torch.int64], pages.ref, DTYPES[dtype], pages.heads, pages.head_dim, _whole(path, T, "path", dev),
                                  _whole(slots, T, "slots", dev), _whole(cu_new, R + 1, "cu_new", dev),
                                  _values(k_pages, pages.seen, "k_pages", dev), _values(v_pages, pages.seen, "v_pages", dev), stream),
           "stem_tree_commit")
