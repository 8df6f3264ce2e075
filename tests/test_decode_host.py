"""Host side of include/stem_decode.h, without a GPU: exported symbols, rotary frequencies, refusals before anything could be
launched, and the binding's own checks.  (Runs against the library, and once more against a build with sanitizers.)"""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import Rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, NO, SPACE = sb.STEM_ERR_INVALID_ARG, sb.STEM_ERR_UNSUPPORTED, sb.STEM_ERR_WORKSPACE
P = 0x1000                                             # an address that nothing looks at


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "stem_decode.h")).read()
    declared = set(re.findall(r"^\s*(?:int|const char\*)\s+(stem_\w+)\s*\(", header, flags=re.M))
    assert declared == set(db.EXPORTED)
    L = ctypes.CDLL(sb.library_path())
    for name in declared:
        assert hasattr(L, name), name


def plain_frequencies(r, theta, kind, factor, trained, low, high):
    f = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if kind == "linear":
        return [x / factor for x in f]
    if kind == "ntk":
        return [(theta * factor ** (r / (r - 2))) ** (-2.0 * i / r) for i in range(r // 2)]
    if kind == "bands":
        out = []
        for x in f:
            length = 2 * math.pi / x                   # of one turn, in tokens
            if length < trained / high:
                out.append(x)
            elif length > trained / low:
                out.append(x / factor)
            else:
                y = (trained / length - low) / (high - low)
                out.append((1 - y) * x / factor + y * x)
        return out
    if kind == "yarn":
        lo = max(math.floor(r * math.log(trained / (2 * math.pi * high)) / (2 * math.log(theta))), 0)
        hi = min(math.ceil(r * math.log(trained / (2 * math.pi * low)) / (2 * math.log(theta))), r - 1)
        out = []
        for i, x in enumerate(f):
            y = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            out.append(x / factor * y + x * (1 - y))
        return out
    return f


@pytest.mark.parametrize("kind,low,high", [("none", 1, 4), ("linear", 1, 4), ("ntk", 1, 4), ("yarn", 1, 32), ("bands", 1, 4)])
@pytest.mark.parametrize("r,theta", [(128, 500000.0), (64, 10000.0), (6, 1e6), (256, 150000.0)])
def test_frequencies(kind, low, high, r, theta):
    turns, factor = db.stem_rotary_frequencies(r, theta, kind, 8.0, 8192.0, low, high)
    want = torch.tensor(plain_frequencies(r, theta, kind, 8.0, 8192.0, low, high), dtype=torch.float64) / (2 * math.pi)
    assert turns.shape == want.shape and ((turns - want).abs() <= 1e-13 * want).all()
    assert factor == (pytest.approx(0.1 * math.log(8.0) + 1.0, rel=1e-15) if kind == "yarn" else 1.0)


def test_frequencies_refused():
    for args, status in (((7, 1e4), BAD), ((0, 1e4), BAD), ((2048, 1e4), NO), ((64, 1.0), BAD), ((64, math.nan), BAD),
                         ((64, 1e4, "linear", 0.5), BAD), ((64, 1e4, "linear", math.inf), BAD), ((2, 1e4, "ntk", 2.0), BAD),
                         ((64, 1e4, "yarn", 2.0, 0.0), BAD), ((64, 1e4, "bands", 2.0, 100.0, 4.0, 4.0), BAD),
                         ((64, 1e4, "bands", 2.0, 100.0, 0.0, 4.0), BAD)):
        with pytest.raises(sb.StemError) as e:
            db.stem_rotary_frequencies(*args)
        assert e.value.status == status, args
    with pytest.raises(ValueError):
        db.stem_rotary_frequencies(64, 1e4, "cubic")
    assert db.lib().stem_rotary_frequencies(64, 1e4, None, None, None) == BAD


def rotary_shape(**kw):
    c = db.stem_rotary_shape(db.STEM_BF16, 10, 4, 2, 128, 128, db.STEM_ROTARY_HALF, 512, 128, 256, 128, 512, 128, 256, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rotary(c, q=P, k=P, pos=P, turns=P, factor=1.0, backward=0, q_out=P, k_out=P):
    return db.lib().stem_rotary(ctypes.byref(c) if c is not None else None, q, k, pos, turns, factor, backward, q_out, k_out, None)


def test_rotary_of_no_values_is_refused():
    for wrong in (0, 63):
        with pytest.raises(sb.StemError):
            Rotary(64, wrong, device="cpu")
    assert Rotary(64, device="cpu").rotary_dim == 64
    with pytest.raises(ValueError):                    # positions of other heads than those that come
        Rotary(128, device="cpu").apply(torch.zeros(3, 2, 64, dtype=torch.bfloat16), None, torch.zeros(3, dtype=torch.int32))


def test_rotary_refusals():
    for kw, status in ((dict(dtype=3), BAD), (dict(tokens=-1), BAD), (dict(tokens=(1 << 24) + 1), NO), (dict(tokens=1 << 24), NO),
                       (dict(num_q_heads=-1), BAD), (dict(num_q_heads=0, num_kv_heads=0), BAD), (dict(num_q_heads=70000), NO),
                       (dict(head_dim=0), BAD), (dict(head_dim=100), BAD), (dict(head_dim=2048), NO),
                       (dict(rotary_dim=0), BAD), (dict(rotary_dim=63), BAD), (dict(rotary_dim=130), BAD), (dict(layout=2), BAD),
                       (dict(q_stride_token=100), BAD), (dict(q_stride_head=132), BAD), (dict(k_stride_token=64), BAD),
                       (dict(q_out_stride_token=516), BAD), (dict(k_out_stride_head=0), BAD), (dict(q_stride_token=1024), BAD)):
        c = rotary_shape(**kw)
        assert rotary(c) == status, kw                 # (the last one: in place with other strides)
    c = rotary_shape()
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(turns=None), dict(q_out=None), dict(k_out=None), dict(q=P + 8),
               dict(k_out=P + 2), dict(pos=P + 2), dict(turns=P + 4), dict(factor=math.nan), dict(factor=math.inf),
               dict(backward=2)):
        assert rotary(c, **kw) == BAD, kw
    assert rotary(None) == BAD
    assert rotary(rotary_shape(tokens=0)) == sb.STEM_OK
    assert rotary(rotary_shape(tokens=0, num_q_heads=0), q=None, q_out=None) == sb.STEM_OK
    assert rotary(rotary_shape(tokens=0, num_kv_heads=0), k=None, k_out=None) == sb.STEM_OK


def pages(**kw):
    c = db.stem_pages(16, 100, 16 * 256, 256, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(c, p, q=P, k=P, v=P, pos=P, slots=P, turns=P, q_out=P, kp=P, vp=P):
    return db.lib().stem_rotary_append(ctypes.byref(c), ctypes.byref(p) if p is not None else None, q, k, v, pos, slots, turns, 1.0,
                                       q_out, kp, vp, None)


BAD_PAGES = ((dict(page_size=0), BAD), (dict(page_size=8), NO), (dict(page_size=48), NO), (dict(page_size=512), NO),
             (dict(num_pages=-1), BAD), (dict(num_pages=1 << 28), NO), (dict(stride_page=64), BAD), (dict(stride_page=4100), BAD),
             (dict(stride_token=64), BAD), (dict(stride_token=132), BAD), (dict(stride_head=100), BAD))


def test_append_refusals():
    c = rotary_shape(tokens=0)
    assert append(c, pages()) == sb.STEM_OK
    c = rotary_shape()
    for kw, status in BAD_PAGES:
        assert append(c, pages(**kw)) == status, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(v=P + 8), dict(pos=None), dict(slots=None), dict(slots=P + 1),
               dict(turns=None), dict(q_out=None), dict(kp=None), dict(vp=None), dict(kp=P + 8)):
        assert append(c, pages(), **kw) == BAD, kw
    assert append(c, None) == BAD
    assert append(rotary_shape(num_kv_heads=0), pages()) == BAD


def table_shape(**kw):
    c = db.stem_table_shape(8, 16, 100, 20, 64, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_table_refusals():
    L, n = db.lib(), ctypes.c_size_t()
    for kw, status in ((dict(requests=0), BAD), (dict(requests=65537), NO), (dict(page_size=0), BAD), (dict(page_size=24), NO),
                       (dict(num_pages=0), BAD), (dict(num_pages=1 << 27), NO), (dict(pages_per_request=0), BAD),
                       (dict(requests=65536, pages_per_request=1 << 15), NO), (dict(token_capacity=-1), BAD),
                       (dict(position_offset=-1), BAD), (dict(position_offset=(1 << 31) - 100), NO)):
        c = table_shape(**kw)
        assert L.stem_block_table_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == status, kw
        assert L.stem_block_table(ctypes.byref(c), *[P] * 12, 1 << 30, None) == status, kw
    c = table_shape()
    assert L.stem_block_table_workspace_bytes(None, ctypes.byref(n)) == BAD
    assert L.stem_block_table_workspace_bytes(ctypes.byref(c), None) == BAD
    assert L.stem_block_table_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == sb.STEM_OK and n.value >= 2 * 4 * 8
    for i in range(12):                                # new_lens (1) may be missing
        args = [P] * 12
        args[i] = None
        if i != 1:
            assert L.stem_block_table(ctypes.byref(c), *args, n.value, None) == BAD, i
        args[i] = P + 2
        assert L.stem_block_table(ctypes.byref(c), *args, n.value, None) == BAD, i
    assert L.stem_block_table(ctypes.byref(c), *[P] * 12, n.value - 1, None) == SPACE


def prefix_shape(**kw):
    c = db.stem_prefix_shape(db.STEM_BF16, 8, 2, 128, 3, 3, 1, 1000, 64, 4, 1024, 128, 256, 128, pages())
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def prefix(c, q=P, pk=P, pv=P, kp=P, vp=P, table=P, lens=P, cu=P, scale=0.1, out=2 * P, lse=P, ws=P, size=1 << 40):
    return db.lib().stem_prefix_attn(ctypes.byref(c), q, pk, pv, kp, vp, table, lens, cu, scale, out, lse, ws, size, None)


def test_prefix_refusals():
    L, n = db.lib(), ctypes.c_size_t()
    bad = [(dict(dtype=db.STEM_FP32), BAD), (dict(num_q_heads=0), BAD), (dict(num_kv_heads=3), BAD), (dict(head_dim=96), NO),
           (dict(head_dim=0), BAD), (dict(requests=0), BAD), (dict(requests=65537), NO), (dict(tokens=-1), BAD),
           (dict(tokens=1 << 28), NO), (dict(max_new=0), BAD), (dict(max_new=1 << 29), NO), (dict(prefix_len=-1), BAD),
           (dict(max_suffix=-1), BAD), (dict(max_suffix=65), BAD), (dict(pages_per_request=0), BAD), (dict(q_stride_token=64), BAD),
           (dict(q_stride_head=132), BAD), (dict(prefix_stride_token=64), BAD), (dict(prefix_stride_token=1 << 27), NO),
           (dict(requests=65536, pages_per_request=1 << 15), NO), (dict(pages=pages(stride_token=1 << 27)), NO)]
    bad += [(dict(pages=pages(**kw)), status) for kw, status in BAD_PAGES]
    for kw, status in bad:
        c = prefix_shape(**kw)
        assert L.stem_prefix_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == status, kw
        assert prefix(c) == status, kw
    assert L.stem_prefix_attn_workspace_bytes(None, ctypes.byref(n)) == BAD
    assert L.stem_prefix_attn_workspace_bytes(ctypes.byref(prefix_shape()), None) == BAD
    c = prefix_shape()
    for kw in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P), dict(lse=P + 2), dict(pk=None), dict(pv=None),
               dict(pv=P + 8), dict(kp=None), dict(vp=P + 8), dict(table=None), dict(table=P + 2), dict(lens=None), dict(lens=P + 2),
               dict(cu=P + 2), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(ws=None),
               dict(ws=P + 8)):
        assert prefix(c, **kw) == BAD, kw
    assert prefix(prefix_shape(tokens=4), cu=None) == BAD          # one token per request, and a row of none
    assert prefix(prefix_shape(tokens=0)) == sb.STEM_OK
    assert prefix(prefix_shape(tokens=0, prefix_len=0), pk=None, pv=None) == sb.STEM_OK
    assert prefix(prefix_shape(tokens=0, max_suffix=0), kp=None, vp=None, table=None, lens=None) == sb.STEM_OK


@pytest.mark.skipif(not (os.path.exists(sb.library_path()) and hasattr(ctypes.CDLL(sb.library_path()), "stem_test_prefix_plan")),
                    reason="needs the host-only build")
def test_prefix_plan_covers_everything_within_its_workspace():
    L = ctypes.CDLL(sb.library_path())
    out = (ctypes.c_int64 * 10)()
    some = [1, 2, 3, 7, 16, 17, 33, 64, 100, 1000, 30000]
    for d in (64, 128, 256):
        for hq, hkv in ((1, 1), (32, 8), (28, 4), (8, 1), (64, 1)):
            for tokens in (1, 2, 5, 16, 64, 100, 4096):
                for L_, S in [(0, 64), (1, 0), *[(x, 64) for x in some], *[(131072, 20 * x) for x in some]]:
                    W = max(1, -(-S // 16))
                    c = prefix_shape(head_dim=d, num_q_heads=hq, num_kv_heads=hkv, tokens=tokens, requests=min(tokens, 64), max_new=7,
                                     prefix_len=L_, max_suffix=S, pages_per_request=W, q_stride_head=d, q_stride_token=hq * d,
                                     prefix_stride_head=d, prefix_stride_token=hkv * d,
                                     pages=pages(stride_page=16 * hkv * d, stride_token=hkv * d, stride_head=d))
                    for units in (256, 304, 32):
                        assert L.stem_test_prefix_plan(ctypes.byref(c), units, out) == sb.STEM_OK
                        tile, tiles, splits, keys, own, owns, parts, ml, size, small = list(out)
                        rows = tokens * (hq // hkv)
                        assert tile * (tiles - 1) < rows <= tile * tiles
                        assert own * (owns - 1) < min(7 * (hq // hkv), rows) <= own * owns      # no request has more rows than there are
                        if small:                      # one workgroup per request and KV head, without parts
                            assert splits == parts == 0 and owns == 1 and own == 16 and size >= 16
                            continue
                        if L_:
                            assert keys % 32 == 0 and keys * (splits - 1) < L_ <= keys * splits
                        else:
                            assert splits == 0
                        assert (parts >= 1) == (S > 0) and parts <= 64
                        n = (splits + parts) * hkv * rows
                        assert ml >= 4 * n * d and size >= ml + 8 * n and ml % 256 == 0
    assert L.stem_test_prefix_plan(ctypes.byref(prefix_shape()), 0, out) == sb.STEM_ERR_HIP


def test_binding_checks_its_tensors(monkeypatch):
    """On CPU tensors, with a current device that none of them is on."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(sb, "_raw_stream", lambda dev: 0)
    q, k = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    shape = db.RotaryShape.from_tensors(q, k, 64)
    assert (shape.c.num_q_heads, shape.c.num_kv_heads, shape.c.q_stride_token, shape.c.k_out_stride_token) == (4, 2, 256, 128)
    pos, turns = torch.zeros(5, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    for args, what in (((q[:4], k, pos, turns), "q is not"), ((q.half(), k, pos, turns), "q is not"),
                       ((q.transpose(0, 1).contiguous().transpose(0, 1), k, pos, turns), "q is not"),
                       ((None, k, pos, turns), "q is missing"), ((q, k, pos, turns), "q is not on the current device")):
        with pytest.raises(ValueError, match=what):
            db.stem_rotary(shape, *args, 1.0, q, k)
    for given, what in (((q.double(), k), "not supported"), ((q, k[:4]), "go with"), ((q[0], k), "tokens, heads"),
                        ((q[..., ::2], k), "contiguous"), ((None, None), "needed")):
        with pytest.raises(ValueError, match=what):
            db.RotaryShape.from_tensors(*given, 64)
    with pytest.raises(ValueError, match="layout"):
        db.RotaryShape.from_tensors(q, k, 64, "third")
    kp = torch.zeros(7, 16, 2, 64, dtype=torch.bfloat16)
    pages_ = db.PageShape.from_tensors(kp, kp.clone())
    assert (pages_.c.page_size, pages_.c.num_pages, pages_.c.stride_page) == (16, 7, 16 * 128)
    with pytest.raises(ValueError):
        db.PageShape.from_tensors(kp, kp.half())
    table = torch.zeros(5, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        db.PrefixShape.from_tensors(q.half(), None, pages_, table, 1, 48)
    with pytest.raises(ValueError):
        db.PrefixShape.from_tensors(q, None, None, 5, 1, 0)
    one = db.PrefixShape.from_tensors(q[:1], k[:1], None, 1, 1, 0)       # strides of single rows and heads do not matter
    assert one.c.prefix_stride_token == 128 and one.c.requests == 1
    with pytest.raises(ValueError, match="int32"):
        db._whole(pos.long(), 5, "x", 0)
    with pytest.raises(ValueError, match="at least"):
        db._whole(pos, 6, "x", 0)
