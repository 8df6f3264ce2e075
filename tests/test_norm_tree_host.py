"""Host side of include/stem_norm.h and include/stem_tree.h, without a GPU: exported symbols, refusals before anything could be launched, the
split of the attention, and the bindings' own checks.  (Runs against the library, and once more against a build with sanitizers.)"""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import norm_binding as nb
from paper_2603_06274_amd import tree_binding as tb
from paper_2603_06274_amd.decode import PagedCache
from paper_2603_06274_amd.norm import NormRotary

from test_decode_host import BAD, BAD_PAGES, NO, P, ROOT, SPACE, pages, prefix_shape, rotary_shape

OK = sb.STEM_OK
BF = torch.bfloat16


@pytest.mark.parametrize("header,binding", [("stem_norm.h", nb), ("stem_tree.h", tb)])
def test_library_exports_every_declared_symbol(header, binding):
    text = open(os.path.join(ROOT, "include", header)).read()
    declared = set(re.findall(r"^\s*(?:int|const char\*)\s+(stem_\w+)\s*\(", text, flags=re.M))
    assert declared == set(binding.EXPORTED)
    L = ctypes.CDLL(sb.library_path())
    for name in declared:
        assert hasattr(L, name), name


def ref(c):
    return ctypes.byref(c) if c is not None else None


# --- norms ------------------------------------------------------------------------------------------------

def norm(**kw):
    n = nb.stem_head_norm(P, P, db.STEM_BF16, 0.0, 1e-6)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def forward(c, n=norm(), q=P, k=P, pos=P, turns=P, factor=1.0, q_out=P, k_out=P):
    return nb.lib().stem_norm_rotary(ref(c), ref(n), q, k, pos, turns, factor, q_out, k_out, None)


def append(c, p, n=norm(), q=P, k=P, v=P, pos=P, slots=P, turns=P, factor=1.0, q_out=P, kp=P, vp=P):
    return nb.lib().stem_norm_rotary_append(ref(c), ref(n), ref(p), q, k, v, pos, slots, turns, factor, q_out, kp, vp, None)


def backward(c, n=norm(), q=P, k=P, pos=P, turns=P, factor=1.0, gq=2 * P, gk=2 * P, dq=3 * P, dk=3 * P, dqw=P, dkw=P, ws=P, size=1 << 40):
    return nb.lib().stem_norm_rotary_backward(ref(c), ref(n), q, k, pos, turns, factor, gq, gk, dq, dk, dqw, dkw, ws, size, None)


def space(c):
    n = ctypes.c_size_t()
    return nb.lib().stem_norm_rotary_backward_workspace_bytes(ref(c), ctypes.byref(n)), n.value


BAD_ROWS = ((dict(dtype=3), BAD), (dict(tokens=-1), BAD), (dict(tokens=1 << 24), NO), (dict(num_q_heads=-1), BAD),
            (dict(num_q_heads=0, num_kv_heads=0), BAD), (dict(num_q_heads=70000), NO), (dict(head_dim=0), BAD), (dict(head_dim=100), BAD),
            (dict(head_dim=2048), NO), (dict(rotary_dim=0), BAD), (dict(rotary_dim=63), BAD), (dict(rotary_dim=130), BAD), (dict(layout=2), BAD),
            (dict(q_stride_token=100), BAD), (dict(q_stride_head=132), BAD), (dict(k_stride_token=64), BAD), (dict(q_out_stride_token=516), BAD))
BAD_NORMS = (None, norm(q_weight=P + 8), norm(k_weight=P + 2), norm(weight_dtype=3), norm(weight_dtype=-1), norm(weight_offset=math.nan),
             norm(weight_offset=math.inf), norm(eps=0.0), norm(eps=-1e-6), norm(eps=math.nan), norm(eps=math.inf), norm(eps=1e-40))


def test_norm_refusals():
    for kw, status in BAD_ROWS:
        c = rotary_shape(**kw)
        assert forward(c) == append(c, pages()) == backward(c) == status, kw
        assert space(c)[0] == status, kw
    assert forward(None) == append(None, pages()) == backward(None) == space(None)[0] == BAD
    c = rotary_shape()
    for n in BAD_NORMS:
        assert forward(c, n) == append(c, pages(), n) == backward(c, n) == BAD
    for factor in (math.nan, math.inf):
        assert forward(c, factor=factor) == append(c, pages(), factor=factor) == backward(c, factor=factor) == BAD
    for kw in (dict(k_out_stride_head=0), dict(k_out_stride_token=132)):
        assert forward(rotary_shape(**kw)) == backward(rotary_shape(**kw)) == BAD, kw
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(turns=None), dict(q_out=None), dict(k_out=None), dict(q=P + 8),
               dict(k_out=P + 2), dict(pos=P + 2), dict(turns=P + 4)):
        assert forward(c, **kw) == BAD, kw
    assert forward(rotary_shape(q_stride_token=1024)) == BAD       # in place with other strides
    assert forward(rotary_shape(k_out_stride_token=512)) == BAD


def test_norm_append_refusals():
    c = rotary_shape()
    for kw, status in BAD_PAGES:
        assert append(c, pages(**kw)) == status, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(v=P + 8), dict(pos=None), dict(slots=None), dict(slots=P + 1),
               dict(turns=None), dict(q_out=None), dict(kp=None), dict(vp=None), dict(kp=P + 8)):
        assert append(c, pages(), **kw) == BAD, kw
    assert append(c, None) == BAD
    assert append(rotary_shape(num_kv_heads=0), pages()) == BAD
    assert append(c, pages(num_pages=0), kp=None, vp=None) == OK   # nowhere to write to


def test_norm_gradients_refusals():
    c = rotary_shape()
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(turns=None), dict(gq=None), dict(gk=None), dict(dq=None), dict(dk=None),
               dict(q=P + 8), dict(gk=P + 2), dict(dq=P + 8), dict(pos=P + 2), dict(turns=P + 4), dict(dqw=P + 2), dict(dkw=P + 1),
               dict(ws=None), dict(ws=P + 8), dict(n=norm(q_weight=None)), dict(n=norm(k_weight=None))):
        assert backward(c, **kw) == BAD, kw
    need = space(c)[1]
    assert need >= 2 * 4 * 128 and backward(c, size=need - 1) == SPACE
    assert backward(rotary_shape(q_stride_token=1024), dq=2 * P) == BAD        # in place of the outputs' gradients, with other strides
    assert nb.lib().stem_norm_rotary_backward_workspace_bytes(ref(c), None) == BAD


def test_norm_of_no_tokens():
    c = rotary_shape(tokens=0)
    assert forward(c, q=None, k=None, pos=None, turns=None, q_out=None, k_out=None) == OK
    assert append(c, pages(), q=None, k=None, v=None, pos=None, slots=None, turns=None, q_out=None) == OK
    nothing = dict(q=None, k=None, pos=None, turns=None, gq=None, gk=None, dq=None, dk=None, ws=None, size=0)
    assert backward(c, dqw=None, dkw=None, **nothing) == OK
    assert space(c) == (OK, 0)


# --- trees ------------------------------------------------------------------------------------------------

def masks(s=None, parents=P, lens=P, cu=P, pos=P, out=P, status=P, **kw):
    c = tb.stem_tree_shape(3, 20, 8, 100)
    for k, v in kw.items():
        setattr(c, k, v)
    return tb.lib().stem_tree_masks(ref(c) if s is None else None, parents, lens, cu, pos, out, status, None)


BAD_SIZES = ((dict(requests=0), BAD), (dict(requests=65537), NO), (dict(tokens=-1), BAD), (dict(max_new=0), BAD), (dict(max_new=1025), NO))


def test_masks_refusals():
    for kw, status in BAD_SIZES + ((dict(position_offset=-1), BAD),):
        assert masks(**kw) == status, kw
    for kw in (dict(s=0), dict(parents=None), dict(lens=None), dict(cu=None), dict(out=None), dict(status=None), dict(parents=P + 2),
               dict(lens=P + 1), dict(cu=P + 2), dict(pos=P + 2), dict(out=P + 4), dict(status=P + 2)):
        assert masks(**kw) == BAD, kw
    assert masks(tokens=0, parents=None, lens=None, cu=None, out=None, status=None) == OK


def attn(c, q=P, pk=P, pv=P, kp=P, vp=P, table=P, lens=P, cu=P, m=P, scale=0.1, out=2 * P, lse=P, ws=P, size=1 << 40):
    return tb.lib().stem_tree_attn(ref(c), q, pk, pv, kp, vp, table, lens, cu, m, scale, out, lse, ws, size, None)


def test_attention_refusals():
    L, n = tb.lib(), ctypes.c_size_t()
    bad = [(dict(dtype=db.STEM_FP32), BAD), (dict(num_kv_heads=3), BAD), (dict(head_dim=96), NO), (dict(requests=0), BAD),
           (dict(tokens=-1), BAD), (dict(max_new=0), BAD), (dict(max_new=1025), NO), (dict(max_suffix=65), BAD),
           (dict(q_stride_token=64), BAD), (dict(prefix_stride_token=1 << 27), NO), (dict(pages=pages(stride_token=1 << 27)), NO)]
    bad += [(dict(pages=pages(**kw)), status) for kw, status in BAD_PAGES]
    for kw, status in bad:
        c = prefix_shape(**kw)
        assert L.stem_tree_attn_workspace_bytes(ref(c), ctypes.byref(n)) == status, kw
        assert attn(c) == status, kw
    assert L.stem_tree_attn_workspace_bytes(None, ctypes.byref(n)) == L.stem_tree_attn_workspace_bytes(ref(prefix_shape()), None) == BAD
    c = prefix_shape()
    for kw in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P), dict(lse=P + 2), dict(pk=None), dict(pv=P + 8), dict(kp=None),
               dict(vp=P + 8), dict(table=None), dict(lens=P + 2), dict(cu=None), dict(cu=P + 2), dict(m=None), dict(m=P + 4),
               dict(scale=0.0), dict(scale=math.nan), dict(ws=None), dict(ws=P + 8)):
        assert attn(c, **kw) == BAD, kw
    assert attn(prefix_shape(tokens=0), m=None) == OK


def accept_shape(**kw):
    c = tb.stem_accept_shape(3, 20, 8, 16, 100, 10, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def accept(c, size=1 << 20, **at):
    args = [P] * 15
    for i, x in at.items():
        args[int(i[1:])] = x
    return tb.lib().stem_tree_accept(ref(c), *args, size, None)


def test_accept_refusals():
    L, n, call = tb.lib(), ctypes.c_size_t(), accept
    for kw, status in BAD_SIZES + ((dict(page_size=0), BAD), (dict(page_size=24), NO), (dict(num_pages=0), BAD), (dict(num_pages=1 << 27), NO),
                                   (dict(pages_per_request=0), BAD), (dict(requests=65536, pages_per_request=1 << 15), NO),
                                   (dict(id_bits=16), BAD)):
        c = accept_shape(**kw)
        assert call(c) == status, kw
        assert L.stem_tree_accept_workspace_bytes(ref(c), ctypes.byref(n)) == status, kw
    assert L.stem_tree_accept_workspace_bytes(None, ctypes.byref(n)) == L.stem_tree_accept_workspace_bytes(ref(accept_shape()), None) == BAD
    assert L.stem_tree_accept_workspace_bytes(ref(accept_shape()), ctypes.byref(n)) == OK
    c = accept_shape()
    for i in range(15):
        assert call(c, **{"a%d" % i: None}) == BAD, i
        assert call(c, **{"a%d" % i: P + 2}) == BAD, i
    for i in (1, 2, 12):                               # ids of 64 bits lie at whole 8 bytes
        assert call(c, **{"a%d" % i: P + 4}) == BAD, i
    assert call(c, size=n.value - 1) == SPACE


def commit(c=accept_shape(), p=pages(), dtype=db.STEM_BF16, heads=2, d=128, path=P, slots=P, cu=P, kp=P, vp=P):
    return tb.lib().stem_tree_commit(ref(c), ref(p), dtype, heads, d, path, slots, cu, kp, vp, None)


def test_commit_refusals():
    for kw, status in BAD_SIZES:
        assert commit(accept_shape(**kw)) == status, kw
    for kw, status in BAD_PAGES:
        assert commit(p=pages(**kw)) == status, kw
    for kw, status in ((dict(dtype=3), BAD), (dict(heads=0), BAD), (dict(d=0), BAD), (dict(d=100), BAD), (dict(d=1032), NO), (dict(c=None), BAD),
                       (dict(p=None), BAD), (dict(path=None), BAD), (dict(slots=None), BAD), (dict(cu=None), BAD), (dict(path=P + 2), BAD),
                       (dict(slots=P + 1), BAD), (dict(cu=P + 2), BAD), (dict(kp=None), BAD), (dict(vp=P + 8), BAD)):
        assert commit(**kw) == status, kw
    wide = pages(stride_token=1 << 26, stride_page=1 << 30, stride_head=1024)
    assert commit(p=wide, heads=32769, d=1024) == NO
    assert commit(p=wide, heads=2 ** 31 - 1, d=1024, dtype=db.STEM_FP32) == NO
    assert commit(accept_shape(tokens=0), path=None, slots=None) == commit(p=pages(num_pages=0), kp=None, vp=None) == OK


HOST_ONLY = os.path.exists(sb.library_path()) and hasattr(ctypes.CDLL(sb.library_path()), "stem_test_tree_plan")
host_only = pytest.mark.skipif(not HOST_ONLY, reason="needs the host-only build")


@host_only
def test_calls_that_are_not_refused():
    c = rotary_shape()
    need = space(c)[1]
    assert forward(c) == forward(c, norm(q_weight=None, k_weight=None)) == OK
    assert append(c, pages()) == append(rotary_shape(num_q_heads=0), pages(), q=None, q_out=None) == OK
    assert backward(c, size=need) == OK
    assert backward(c, dqw=None, dkw=None, ws=None, size=0) == OK  # no weight's gradient wanted
    assert backward(c, n=norm(q_weight=None), dqw=None) == OK
    # the gradients in place of the inputs, or of the outputs' if the strides are the same
    assert backward(c, dq=P, dk=P) == backward(c, dq=2 * P, dk=2 * P) == backward(rotary_shape(q_stride_token=1024), dq=P) == OK
    nothing = dict(q=None, k=None, pos=None, turns=None, gq=None, gk=None, dq=None, dk=None, ws=None, size=0)
    assert backward(rotary_shape(tokens=0), **nothing) == OK       # (the sums become 0)
    assert masks() == masks(pos=None) == masks(max_new=1024) == OK
    assert accept(accept_shape()) == accept(accept_shape(id_bits=32)) == OK
    for i in (1, 2, 12):
        assert accept(accept_shape(id_bits=32), **{"a%d" % i: P + 4}) == OK, i
    assert accept(accept_shape(), size=256) == accept(accept_shape(tokens=0), a0=None, a1=None, a2=None, a11=None) == OK
    wide = pages(stride_token=1 << 26, stride_page=1 << 30, stride_head=1024)
    assert commit() == commit(p=wide, heads=32768, d=1024) == OK   # 64 MiB of K per token


@host_only
def test_the_split_covers_all_own_keys_within_its_workspace():
    L = ctypes.CDLL(sb.library_path())
    out = (ctypes.c_int64 * 10)()
    for d in (64, 128, 256):
        for hq, hkv in ((1, 1), (32, 8), (28, 4), (8, 1)):
            G = hq // hkv
            for requests, tokens, max_new in ((1, 1, 1), (3, 40, 17), (64, 64, 1), (48, 3000, 128), (2, 2048, 1024), (500, 900, 64)):
                for suffix in (16, 400, 2048, 33000, 1 << 20):
                    for prefix_len in (0, 500, 65535):
                        c = prefix_shape(head_dim=d, num_q_heads=hq, num_kv_heads=hkv, tokens=tokens, requests=requests, max_new=max_new,
                                         prefix_len=prefix_len, max_suffix=suffix, pages_per_request=-(-suffix // 16), q_stride_head=d,
                                         q_stride_token=hq * d, prefix_stride_head=d, prefix_stride_token=hkv * d,
                                         pages=pages(stride_page=16 * hkv * d, stride_token=hkv * d, stride_head=d, num_pages=1 << 20))
                        assert L.stem_test_tree_plan(ctypes.byref(c), 256, out) == OK
                        tile, tiles, splits, least, prefix_splits, slots, ml, size, small, groups = list(out)
                        own = min(max_new * G, tokens * G)
                        assert tile * (tiles - 1) < own <= tile * tiles
                        if small:                  # one launch, a workgroup for each row tile of a request
                            assert splits == prefix_splits == 0 and requests * tiles * hkv <= 512 and prefix_len + suffix <= 1536
                            assert tile == (16 if own <= 16 and d != 256 else 32 if d == 256 else 64) or (tile, d) == (16, 64)
                            continue
                        assert 1 <= splits <= 64 and slots >= min(requests * tiles, requests + tokens * G // tile)
                        n = (splits + prefix_splits) * hkv * tokens * G
                        assert ml >= 4 * n * d and size >= ml + 8 * n and ml % 256 == 0 and groups >= slots * hkv * splits
                        for length in {1, 127, 129, suffix // 3 + 1, suffix}:
                            if length > suffix:
                                continue
                            keys, parts = L.stem_test_split_keys(length, splits, least), L.stem_test_parts(length, splits, least)
                            assert keys % 128 == 0 and keys >= least and parts <= splits and keys * (parts - 1) < length <= keys * parts
    for requests, tokens, max_new in ((1, 1, 1), (3, 3000, 1024)):
        big = prefix_shape(requests=requests, max_new=max_new, max_suffix=2 ** 31 - 2 ** 14, pages_per_request=1 << 27, tokens=tokens)
        assert L.stem_test_tree_plan(ctypes.byref(big), 256, out) == OK
        splits, least = list(out)[2:4]
        assert L.stem_test_split_keys(2 ** 31 - 2 ** 14, splits, least) * splits < 2 ** 31 - 4 * 256       # (what a walk looks ahead)


# --- bindings ---------------------------------------------------------------------------------------------

@pytest.fixture
def here(monkeypatch):
    """Calls whose current device is that of tensors on the host."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(sb, "_raw_stream", lambda dev: 0)


def whole(*sizes, dtype=torch.int32):
    return torch.zeros(*sizes, dtype=dtype)


def test_weights_that_cannot_be_used():
    w = torch.ones(64)
    for given in ((w.view(8, 8), None), (torch.ones(128)[::2], None), (w.double(), None), (w, w.half()), (w, torch.ones(72))):
        with pytest.raises(ValueError):
            nb.HeadNorm(*given)
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-39), dict(eps=1e39),
               dict(weight_offset=math.nan), dict(weight_offset=math.inf)):
        with pytest.raises(ValueError):
            nb.HeadNorm(w, w, **kw)
    with pytest.raises(ValueError):
        NormRotary(128, w, w, device="cpu")            # weights of other heads
    with pytest.raises(ValueError):
        NormRotary(64, torch.ones(65)[1:], None, device="cpu")         # at no whole 16 bytes
    assert NormRotary(64, w, None, device="cpu").norm.head_dim == NormRotary.none(64, w, device="cpu").norm.head_dim == 64
    assert NormRotary(64, None, None, device="cpu").norm.head_dim is None


def test_norm_binding_checks_its_tensors(here):
    r = NormRotary(64, torch.ones(64), torch.ones(64), device="cpu")
    q, k, pos = torch.zeros(5, 4, 64, dtype=BF), torch.zeros(5, 2, 64, dtype=BF), whole(5)
    shape = r._shape(q, k, q, k)

    def call(q=q, k=k, pos=pos, turns=r.turns, q_out=q, k_out=k, n=r.norm):
        nb.stem_norm_rotary(shape, n, q, k, pos, turns, 1.0, q_out, k_out)

    for kw, what in ((dict(q=q[:4]), "q is not"), (dict(k=k.half()), "k is not"), (dict(q=None), "q is missing"), (dict(q_out=None), "q_out"),
                     (dict(k_out=k[:, :1]), "k_out"), (dict(pos=pos[:4]), "positions"), (dict(pos=pos.long()), "positions"),
                     (dict(turns=r.turns.float()), "turns"), (dict(n=nb.HeadNorm(torch.ones(72), None)), "weights of 72")):
        with pytest.raises(ValueError, match=what):
            call(**kw)
    with pytest.raises(TypeError):
        r.backward(q, k, pos)
    with pytest.raises(ValueError, match="carry no gradients"):
        r.apply(q.requires_grad_(), k, pos, q_out=torch.zeros_like(q))
    with pytest.raises(ValueError):
        r.apply(torch.zeros(5, 4, 128, dtype=BF), None, pos)       # heads of other sizes
    sums, ws = whole(64, dtype=torch.float32), whole(1 << 20, dtype=torch.uint8)
    q = q.detach()

    def grads(gq=q, gk=k, dq=q, dk=k, dqw=sums, dkw=sums, ws=ws):
        nb.stem_norm_rotary_backward(shape, r.norm, q, k, pos, r.turns, 1.0, gq, gk, dq, dk, dqw, dkw, ws)

    for kw, what in ((dict(gq=None), "grad_q"), (dict(gk=k.half()), "grad_k"), (dict(dq=q[:3]), "q_grad"), (dict(dk=None), "k_grad"),
                     (dict(dqw=sums[:60]), "q_weight_grad"), (dict(dkw=sums.half()), "k_weight_grad"), (dict(ws=sums), "workspace")):
        with pytest.raises(ValueError, match=what):
            grads(**kw)
    with pytest.raises(sb.StemError):
        grads(ws=ws[:256])
    for f in (lambda: call(q), lambda: grads()):       # of another device than the current one
        torch.cuda.current_device = lambda: 0
        with pytest.raises(ValueError, match="current device"):
            f()


def test_tree_binding_checks_its_tensors(here):
    R, T, W = 3, 20, 2
    shape = tb.TreeShape(R, T, 100)
    good = dict(parents=whole(T), lens=whole(R), cu_new=whole(R + 1), positions=whole(T), masks=whole(T, W, dtype=torch.int64), status=whole(1))
    for kw, what in ((dict(parents=whole(T - 1)), "parents"), (dict(lens=whole(R, dtype=torch.int64)), "lens"), (dict(cu_new=whole(R)), "cu_new"),
                     (dict(positions=whole(T - 1)), "positions"), (dict(masks=whole(T, 1, dtype=torch.int64)), "masks"),
                     (dict(masks=whole(T, W)), "masks"), (dict(status=None), "status"), (dict(parents=None), "parents")):
        with pytest.raises(ValueError, match=what):
            tb.stem_tree_masks(shape, *{**good, **kw}.values())
    shape, n = tb.AcceptShape(R, T, 100, 16, 30, 5), dict(dtype=torch.int64)
    good = dict(parents=whole(T), draft_ids=whole(T, **n), target_ids=whole(T, **n), cu_new=whole(R + 1), lens=whole(R), ring_state=whole(2),
                ring=whole(30), table=whole(R, 5), lens_out=whole(R), ring_state_out=whole(2), accepted=whole(R), path=whole(T),
                next_ids=whole(R, **n), status=whole(2), workspace=whole(256, dtype=torch.uint8))
    for kw, what in ((dict(draft_ids=whole(T, dtype=torch.int16)), "not supported"), (dict(target_ids=whole(T)), "target_ids"),
                     (dict(next_ids=whole(R)), "next_ids"), (dict(ring=whole(29)), "ring"), (dict(table=whole(R, 6)), "table"),
                     (dict(path=whole(T - 1)), "path"), (dict(accepted=whole(R - 1)), "accepted"), (dict(status=whole(1)), "status"),
                     (dict(workspace=whole(256)), "workspace"), (dict(ring_state_out=whole(1)), "ring_state_out")):
        with pytest.raises(ValueError, match=what):
            tb.stem_tree_accept(shape, *{**good, **kw}.values())
    with pytest.raises(sb.StemError):
        tb.stem_tree_accept(shape, *{**good, "workspace": whole(255, dtype=torch.uint8)}.values())
    kp = whole(30, 16, 2, 64, dtype=BF)
    at = db.PageShape.from_tensors(kp, kp.clone())
    good = dict(path=whole(T), slots=whole(T), cu_new=whole(R + 1), k_pages=kp, v_pages=kp.clone())
    for kw, what in ((dict(path=whole(T - 1)), "path"), (dict(slots=whole(T, **n)), "slots"), (dict(cu_new=whole(R)), "cu_new"),
                     (dict(k_pages=kp[:29]), "k_pages"), (dict(v_pages=kp.half()), "v_pages"), (dict(v_pages=None), "v_pages")):
        with pytest.raises(ValueError, match=what):
            tb.stem_tree_commit(shape, at, *{**good, **kw}.values())


def test_nothing_is_accepted_twice_or_before_a_step(here, monkeypatch):
    calls = []
    monkeypatch.setattr(db, "stem_block_table", lambda *a: calls.append("table"))
    for name in ("stem_tree_accept", "stem_tree_commit"):
        monkeypatch.setattr(tb, name, lambda *a, _n=name: calls.append(_n))
    cache = PagedCache(2, 4, 16, 2, 1, 64, tokens=4, device="cpu")
    x = whole(4)
    for _ in range(2):
        with pytest.raises(RuntimeError):
            cache.accept(x, x, x)
        cache.advance(None, 2)
        with pytest.raises(ValueError):
            cache.accept(x, x.float(), x.float())
        cache.accept(x, x, x)
    assert calls == ["table", "stem_tree_accept", "stem_tree_commit"] * 2
