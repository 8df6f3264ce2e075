"""ctypes binding of the entry points in include/stem_decode.h: rotary positions, block tables, writes into pages, attention to
a shared prefix.

Function names and argument order follow the header.  The shape classes read sizes and strides from tensors once; a call then
checks that the tensors it gets are of that shape's types and sizes and on the current device, and passes their addresses.
Every step runs inside the library's HIP kernels on torch's current stream; there is no fallback.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import warnings
from typing import Optional, Tuple

import torch

from . import binding as sb

STEM_BF16, STEM_FP16, STEM_FP32 = 0, 1, 2
STEM_ROTARY_HALF, STEM_ROTARY_INTERLEAVED = 0, 1
STEM_ROTARY_NONE, STEM_ROTARY_LINEAR, STEM_ROTARY_NTK, STEM_ROTARY_YARN, STEM_ROTARY_BANDS = range(5)

DTYPES = {torch.bfloat16: STEM_BF16, torch.float16: STEM_FP16, torch.float32: STEM_FP32}
LAYOUTS = {"half": STEM_ROTARY_HALF, "interleaved": STEM_ROTARY_INTERLEAVED}
SCALINGS = {"none": STEM_ROTARY_NONE, "linear": STEM_ROTARY_LINEAR, "ntk": STEM_ROTARY_NTK, "yarn": STEM_ROTARY_YARN,
            "bands": STEM_ROTARY_BANDS}

STEM_MAX_HEAD_DIM, MAX_TOKENS, MAX_HEADS = 1024, (1 << 24) - 1, 65535      # of stem_rotary and stem_rotary_append

EXPORTED = ["stem_rotary_frequencies", "stem_rotary", "stem_block_table_workspace_bytes", "stem_block_table",
            "stem_rotary_append", "stem_prefix_attn_workspace_bytes", "stem_prefix_attn"]

_i32, _i64, _f32, _f64, _vp, _sz = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_void_p,
                                    ctypes.c_size_t)


class stem_rotary_scaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("factor", _f64), ("trained_length", _f64), ("low", _f64), ("high", _f64)]


class stem_rotary_shape(ctypes.Structure):
    _fields_ = [(x, _i32) for x in ("dtype", "tokens", "num_q_heads", "num_kv_heads", "head_dim", "rotary_dim", "layout")] + [
        (x, _i64) for x in ("q_stride_token", "q_stride_head", "k_stride_token", "k_stride_head", "q_out_stride_token",
                            "q_out_stride_head", "k_out_stride_token", "k_out_stride_head")]


class stem_table_shape(ctypes.Structure):
    _fields_ = [(x, _i32) for x in ("requests", "page_size", "num_pages", "pages_per_request", "token_capacity",
                                    "position_offset", "max_new")]


class stem_pages(ctypes.Structure):
    _fields_ = [("page_size", _i32), ("num_pages", _i32), ("stride_page", _i64), ("stride_token", _i64), ("stride_head", _i64)]


class stem_prefix_shape(ctypes.Structure):
    _fields_ = [(x, _i32) for x in ("dtype", "num_q_heads", "num_kv_heads", "head_dim", "requests", "tokens", "max_new",
                                    "prefix_len", "max_suffix", "pages_per_request")] + [
        (x, _i64) for x in ("q_stride_token", "q_stride_head", "prefix_stride_token", "prefix_stride_head")] + [
        ("pages", stem_pages)]


_lib = None


def lib() -> ctypes.CDLL:
    """The library that binding.lib() loads, with these entry points' signatures.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = sb.lib()
        rot, tab, pre, pages, size = (ctypes.POINTER(x) for x in (stem_rotary_shape, stem_table_shape, stem_prefix_shape,
                                                                  stem_pages, _sz))
        sigs = {
            "stem_rotary_frequencies": [_i32, _f64, ctypes.POINTER(stem_rotary_scaling), ctypes.POINTER(_f64),
                                        ctypes.POINTER(_f64)],
            "stem_rotary": [rot, _vp, _vp, _vp, _vp, _f32, _i32, _vp, _vp, _vp],
            "stem_block_table_workspace_bytes": [tab, size],
            "stem_block_table": [tab] + [_vp] * 12 + [_sz, _vp],
            "stem_rotary_append": [rot, pages, _vp, _vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _vp],
            "stem_prefix_attn_workspace_bytes": [pre, size],
            "stem_prefix_attn": [pre] + [_vp] * 8 + [_f32, _vp, _vp, _vp, _sz, _vp],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != sb.STEM_OK:
        raise sb.StemError(status, where)


def _need(condition: bool, what: str) -> None:
    if not condition:
        raise ValueError(what)


def _here() -> Tuple[int, int]:
    """The current device, on which a call's tensors have to lie, and the handle of its current stream, to which the call goes."""
    dev = torch.cuda.current_device()
    return dev, sb._stream() if sb._raw_stream is None else sb._raw_stream(dev)


def _rows(t: torch.Tensor, name: str) -> Tuple[int, int, int, int, int]:
    """Sizes and strides of [tokens, heads, head_dim] values.  A dimension of one element has no stride that matters: it gets one
    that the library accepts."""
    _need(t.dim() == 3, "%s has to be [tokens, heads, head_dim]" % name)
    T, H, d = t.shape
    _need(d == 1 or t.stride(2) == 1, "%s: the last dimension has to be contiguous" % name)
    return T, H, d, t.stride(0) if T > 1 else H * d if H > 0 else d, t.stride(1) if H > 1 else d


def _dtype(t: torch.Tensor, name: str) -> int:
    _need(t.dtype in DTYPES, "%s: %s is not supported" % (name, t.dtype))
    return DTYPES[t.dtype]


# (These two run for every tensor of every call: conditions first, texts only where one fails.)
def _values(t: Optional[torch.Tensor], like: Optional[tuple], name: str, dev: int) -> Optional[int]:
    """Address of a tensor of values that has to be as `like` says: (shape, strides, dtype)."""
    if like is None:
        return None
    if t is None:
        raise ValueError("%s is missing" % name)
    if t.shape != like[0] or t.dtype is not like[2] or (t.stride() != like[1] and t.numel() > 0):
        raise ValueError("%s is not of the shape's sizes, strides and type" % name)
    if t.get_device() != dev:
        raise ValueError("%s is not on the current device" % name)
    return t.data_ptr()


def _whole(t: Optional[torch.Tensor], n: int, name: str, dev: int, dtype: torch.dtype = torch.int32) -> int:
    """Address of a contiguous tensor of n numbers (or more: what lies behind is not touched)."""
    if t is None or t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError("%s has to be contiguous %s of at least %d elements" % (name, dtype, n))
    if t.get_device() != dev:
        raise ValueError("%s is not on the current device" % name)
    return t.data_ptr()


def _lines(t: Optional[torch.Tensor], n: int, each: int, name: str, dev: int, dtype: torch.dtype = torch.int32) -> int:
    """Address of a contiguous tensor of n lines (or more) of `each` numbers; one of another number of dimensions than two is
    taken for these lines one after the other."""
    s = () if t is None else t.shape
    fit = s[0] >= n and s[1] == each if len(s) == 2 else len(s) > 0 and t.numel() >= n * each
    if not fit or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError("%s has to be contiguous %s of at least %d lines of %d" % (name, dtype, n, each))
    if t.get_device() != dev:
        raise ValueError("%s is not on the current device" % name)
    return t.data_ptr()


try:                                                   # the same three in compiled code, for tensors that are as they have to be
    _tensors = importlib.import_module("._tensors", __package__)
except ModuleNotFoundError:                            # (not built)
    _tensors = None
except ImportError as e:
    _tensors = None
    warnings.warn("tensors are checked in Python, which takes longer: %s" % e, RuntimeWarning)
else:
    _tensors.begin(_values, _whole, _lines)
    _values, _whole, _lines = _tensors.values, _tensors.whole, _tensors.lines


def _seen(t: Optional[torch.Tensor]) -> Optional[tuple]:
    return None if t is None else (t.shape, t.stride(), t.dtype)


def stem_rotary_frequencies(rotary_dim: int, theta: float, scaling: str = "none", factor: float = 1.0,
                            trained_length: float = 0.0, low: float = 1.0, high: Optional[float] = None) -> Tuple[torch.Tensor, float]:
    """(turns float64 CPU tensor [rotary_dim / 2], attention factor) of a scaling method ("none", "linear", "ntk", "yarn", "bands").
    low and high: numbers of turns within the trained length between which the scaling sets in; high None: the method's own, 32 for
    "yarn" and 4 for "bands"."""
    _need(scaling in SCALINGS, "unknown scaling %r" % (scaling,))
    if high is None:
        high = 32.0 if scaling == "yarn" else 4.0
    c = stem_rotary_scaling(SCALINGS[scaling], float(factor), float(trained_length), float(low), float(high))
    out = torch.zeros(max(int(rotary_dim) // 2, 1), dtype=torch.float64)
    af = _f64()
    _check(lib().stem_rotary_frequencies(int(rotary_dim), float(theta), ctypes.byref(c),
                                         ctypes.cast(out.data_ptr(), ctypes.POINTER(_f64)), ctypes.byref(af)),
           "stem_rotary_frequencies")
    return out, af.value


class RotaryShape:
    """Sizes and strides of a rotary call.  q [T, Hq, d], k [T, Hkv, d]; either may be None.  The outputs' strides are those of q_out
    and k_out (None: those of q and k)."""

    def __init__(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], rotary_dim: int, layout: str = "half",
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        _need(q is not None or k is not None, "q or k is needed")
        _need(layout in LAYOUTS, "unknown layout %r" % (layout,))
        first, name = (q, "q") if q is not None else (k, "k")
        dtype, tokens, head_dim = _dtype(first, name), first.shape[0], first.shape[-1]
        least, bits = head_dim, 0                          # the shortest stride, and all strides' bits

        def part(t, name, heads=None):
            nonlocal least, bits
            T, H, d, st, sh = _rows(t, name)
            if t.dtype is not first.dtype or T != tokens or d != head_dim or heads not in (None, H):
                raise ValueError("%s does not go with the others" % name)
            least, bits = min(least, st, sh), bits | st | sh
            return H, st, sh

        Hq, q_st, q_sh = part(q, "q") if q is not None else (0, 0, 0)
        Hkv, k_st, k_sh = part(k, "k") if k is not None else (0, 0, 0)
        _, qo_st, qo_sh = part(q_out, "q_out", Hq) if q_out is not None else (Hq, q_st, q_sh)
        _, ko_st, ko_sh = part(k_out, "k_out", Hkv) if k_out is not None else (Hkv, k_st, k_sh)
        self.c = c = stem_rotary_shape(dtype, tokens, Hq, Hkv, head_dim, int(rotary_dim), LAYOUTS[layout], q_st, q_sh, k_st, k_sh,
                                       qo_st, qo_sh, ko_st, ko_sh)
        self.usable = least >= head_dim and not bits & 7   # what the library asks of strides
        self.q, self.k = _seen(q), _seen(k)
        self.q_out = _seen(q_out) if q_out is not None else self.q
        self.k_out = _seen(k_out) if k_out is not None else self.k
        self.tokens, self.pairs = tokens, c.rotary_dim // 2
        self.ref = ctypes.byref(c)

    @classmethod
    def from_tensors(cls, q, k, rotary_dim: int, layout: str = "half", q_out=None, k_out=None) -> "RotaryShape":
        return cls(q, k, rotary_dim, layout, q_out, k_out)


def stem_rotary(shape: RotaryShape, q, k, positions: torch.Tensor, turns: torch.Tensor, attention_factor: float, q_out, k_out,
                backward: bool = False) -> None:
    dev, stream = _here()
    _check(lib().stem_rotary(shape.ref, _values(q, shape.q, "q", dev), _values(k, shape.k, "k", dev),
                             _whole(positions, shape.tokens, "positions", dev),
                             _whole(turns, shape.pairs, "turns", dev, torch.float64), attention_factor, int(bool(backward)),
                             _values(q_out, shape.q_out, "q_out", dev), _values(k_out, shape.k_out, "k_out", dev),
                             stream), "stem_rotary")


def usable_rows(t: torch.Tensor) -> bool:
    """Whether the library takes the strides and the address of rows [tokens, heads, head_dim]."""
    _, _, d, token, head = _rows(t, "rows") if t.stride(-1) == 1 else (0, 0, 1, 0, 0)
    return min(token, head) >= d and not (token | head) & 7 and not t.data_ptr() & 15


def need_usable_rows(shape: RotaryShape, *rows: Optional[torch.Tensor]) -> None:
    """What the library asks of the rows of a call beyond their sizes: whole 16 bytes, and no row within another."""
    at = 0
    for t in rows:
        if t is not None:
            at |= t.data_ptr()
    if at & 15 or not shape.usable:
        raise ValueError("rows have to begin at whole 16 bytes, %d or more elements apart" % shape.c.head_dim)


class PageShape:
    """Sizes and strides of k_pages and v_pages, both [num_pages, page_size, Hkv, d] with the same strides."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _need(k_pages.dim() == 4 and k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype and
              k_pages.stride() == v_pages.stride(), "k_pages and v_pages have to be alike, [num_pages, page_size, heads, head_dim]")
        _need(k_pages.shape[3] == 1 or k_pages.stride(3) == 1, "k_pages: the last dimension has to be contiguous")
        N, P, H, d = k_pages.shape
        sh = k_pages.stride(2) if H > 1 else d
        st = k_pages.stride(1) if P > 1 else H * sh
        self.c = stem_pages(P, N, k_pages.stride(0) if N > 1 else max(P * st, d), st, sh)
        self.heads, self.head_dim, self.seen = H, d, _seen(k_pages)
        self.ref = ctypes.byref(self.c)

    @classmethod
    def from_tensors(cls, k_pages, v_pages) -> "PageShape":
        return cls(k_pages, v_pages)


def stem_rotary_append(shape: RotaryShape, pages: PageShape, q, k, v, positions: torch.Tensor, slots: torch.Tensor,
                       turns: torch.Tensor, attention_factor: float, q_out, k_pages: torch.Tensor,
                       v_pages: torch.Tensor) -> None:
    dev, stream = _here()
    _need(pages.heads == shape.c.num_kv_heads and pages.head_dim == shape.c.head_dim and
          (shape.k is None or pages.seen[2] == shape.k[2]), "the pages do not go with k")
    _check(lib().stem_rotary_append(shape.ref, pages.ref, _values(q, shape.q, "q", dev), _values(k, shape.k, "k", dev),
                                    _values(v, shape.k, "v", dev), _whole(positions, shape.tokens, "positions", dev),
                                    _whole(slots, shape.tokens, "slots", dev),
                                    _whole(turns, shape.pairs, "turns", dev, torch.float64), attention_factor,
                                    _values(q_out, shape.q_out, "q_out", dev), _values(k_pages, pages.seen, "k_pages", dev),
                                    _values(v_pages, pages.seen, "v_pages", dev), stream), "stem_rotary_append")


class TableShape:
    """Sizes of a block table and of the step that it is brought up to date for; max_new 0: any number of new tokens per request."""

    def __init__(self, requests: int, page_size: int, num_pages: int, pages_per_request: int, token_capacity: int,
                 position_offset: int = 0, max_new: int = 0):
        self.c = stem_table_shape(int(requests), int(page_size), int(num_pages), int(pages_per_request), int(token_capacity),
                                  int(position_offset), int(max_new))
        self.sizes = int(requests), int(num_pages), int(pages_per_request), int(token_capacity)     # what its tensors go by
        self.ref = ctypes.byref(self.c)


def stem_block_table_workspace_bytes(shape: TableShape) -> int:
    n = _sz()
    _check(lib().stem_block_table_workspace_bytes(shape.ref, ctypes.byref(n)), "stem_block_table_workspace_bytes")
    return n.value


def stem_block_table(shape: TableShape, past_lens: torch.Tensor, new_lens: Optional[torch.Tensor], ring_state: torch.Tensor,
                     ring: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, ring_state_out: torch.Tensor,
                     cu_new: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, status: torch.Tensor,
                     workspace: torch.Tensor) -> None:
    dev, stream = _here()
    R, N, W, T = shape.sizes
    _check(lib().stem_block_table(
        shape.ref, _whole(past_lens, R, "past_lens", dev), None if new_lens is None else _whole(new_lens, R, "new_lens", dev),
        _whole(ring_state, 2, "ring_state", dev), _whole(ring, N, "ring", dev),
        _lines(table, R, W, "table", dev), _whole(lens, R, "lens", dev),
        _whole(ring_state_out, 2, "ring_state_out", dev), _whole(cu_new, R + 1, "cu_new", dev),
        _whole(positions, T, "positions", dev), _whole(slots, T, "slots", dev),
        _whole(status, 4, "status", dev), _whole(workspace, 0, "workspace", dev, torch.uint8), workspace.numel(),
        stream), "stem_block_table")


class PrefixShape:
    """Sizes and strides of the attention to a shared prefix.  q [T, Hq, d] (the output has its strides); prefix_k (and prefix_v)
    [L, Hkv, d] or None; pages a PageShape or None, with table [requests, pages_per_request]; without pages, the number of requests
    is given instead of a table."""

    def __init__(self, q: torch.Tensor, prefix_k: Optional[torch.Tensor], pages: Optional[PageShape], table, max_new: int,
                 max_suffix: int):
        T, Hq, d, q_st, q_sh = _rows(q, "q")
        self.c = c = stem_prefix_shape(_dtype(q, "q"), Hq, 0, d, 0, T, int(max_new), 0, int(max_suffix), 0, q_st, q_sh)
        _need(prefix_k is not None or pages is not None, "a prefix or pages are needed")
        if prefix_k is not None:
            L, c.num_kv_heads, dk, c.prefix_stride_token, c.prefix_stride_head = _rows(prefix_k, "prefix_k")
            _need(prefix_k.dtype == q.dtype and dk == d, "prefix_k does not go with q")
            c.prefix_len = L
        if pages is not None:
            _need(pages.seen[2] == q.dtype and pages.head_dim == d and (prefix_k is None or pages.heads == c.num_kv_heads),
                  "the pages do not go with q and the prefix")
            _need(table.dim() == 2, "table has to be [requests, pages_per_request]")
            c.num_kv_heads = pages.heads
            c.requests, c.pages_per_request = table.shape
            c.pages = pages.c
        else:
            _need(int(max_suffix) == 0, "a suffix needs pages")
            c.requests = table if isinstance(table, int) else table.shape[0]
        self.q, self.prefix, self.pages = _seen(q), _seen(prefix_k), pages.seen if pages is not None else None
        self.sizes = c.requests, c.pages_per_request, c.max_suffix > 0, Hq, T                        # what its tensors go by
        self.ref = ctypes.byref(c)

    @classmethod
    def from_tensors(cls, q, prefix_k, pages, table, max_new: int, max_suffix: int) -> "PrefixShape":
        return cls(q, prefix_k, pages, table, max_new, max_suffix)


def need_usable_prefix(shape: PrefixShape, prefix_k, prefix_v, softmax_scale: float) -> None:
    """What stem_prefix_attn asks of the prefix and of the scale."""
    for t, name in ((prefix_k, "prefix_k"), (prefix_v, "prefix_v")):
        if shape.prefix is not None:
            _need(_values(t, shape.prefix, name, prefix_k.get_device()) % 16 == 0, "%s has to begin at whole 16 bytes" % name)
    scale = _f32(softmax_scale).value
    _need(0.0 < scale < math.inf, "%r is no scale in fp32" % softmax_scale)


def stem_prefix_attn_workspace_bytes(shape: PrefixShape) -> int:
    n = _sz()
    _check(lib().stem_prefix_attn_workspace_bytes(shape.ref, ctypes.byref(n)), "stem_prefix_attn_workspace_bytes")
    return n.value


def stem_prefix_attn(shape: PrefixShape, q: torch.Tensor, prefix_k, prefix_v, k_pages, v_pages, table, lens,
                     cu_new: Optional[torch.Tensor], softmax_scale: float, out: torch.Tensor, lse: Optional[torch.Tensor],
                     workspace: torch.Tensor) -> None:
    dev, stream = _here()
    R, W, paged, Hq, T = shape.sizes
    _check(lib().stem_prefix_attn(
        shape.ref, _values(q, shape.q, "q", dev), _values(prefix_k, shape.prefix, "prefix_k", dev),
        _values(prefix_v, shape.prefix, "prefix_v", dev), _values(k_pages, shape.pages, "k_pages", dev) if paged else None,
        _values(v_pages, shape.pages, "v_pages", dev) if paged else None,
        _lines(table, R, W, "table", dev) if paged else None, _whole(lens, R, "lens", dev) if paged else None,
        None if cu_new is None else _whole(cu_new, R + 1, "cu_new", dev), softmax_scale,
        _values(out, shape.q, "out", dev), None if lse is None else _lines(lse, Hq, T, "lse", dev, torch.float32),
        _whole(workspace, 0, "workspace", dev, torch.uint8), workspace.numel(), stream), "stem_prefix_attn")
