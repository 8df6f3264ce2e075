"""Halves of a head that do not begin at whole chunks of 16 bytes: heads of every number of lanes, halves that end in every place of a
lane's values, and new tokens' rows in pages, beside values that are not normalised (V) in the same waves."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import norm_binding as nb

import norm_util as nu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
EPS = 2.0 ** -20
SIZES = [(8, 6), (16, 14), (24, 22), (64, 2), (64, 18), (64, 30), (64, 62), (96, 24), (128, 4), (128, 50), (128, 126), (200, 198), (256, 250),
         (512, 510), (1024, 34), (1024, 1022)]


def rows(g, n, h, d, dtype):
    return torch.randn(n, h, d, generator=g).to(dtype)


def ws_of(g, d):
    return [1 + 0.2 * torch.randn(d, generator=g) for _ in range(2)]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("d,rot", SIZES)
def test_values_and_gradients(dtype, d, rot):
    g = torch.Generator().manual_seed(d + rot)
    T, Hq, Hkv = 37, 3, 2
    q, k, gq, gk = (rows(g, T, h, d, dtype) for h in (Hq, Hkv, Hq, Hkv))
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0)
    ws = ws_of(g, d)
    norm = nb.HeadNorm(*(w.to(DEV) for w in ws), EPS, 0.0)
    x = [t.to(DEV) for t in (q, k)]
    shape = db.RotaryShape.from_tensors(*x, rot, "half")
    out = [torch.full_like(t, float("nan")) for t in x]
    nb.stem_norm_rotary(shape, norm, *x, pos.to(DEV), turns.to(DEV), factor, *out)
    grads, sums = [torch.full_like(t, float("nan")) for t in x], [torch.full((d,), float("nan"), device=DEV) for _ in ws]
    space = torch.full((nb.stem_norm_rotary_backward_workspace_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    nb.stem_norm_rotary_backward(shape, norm, *x, pos.to(DEV), turns.to(DEV), factor, gq.to(DEV), gk.to(DEV), *grads, *sums, space)
    for t, gy, w, y, dx, dw in zip((q, k), (gq, gk), ws, out, grads, sums):
        args = t, w, 0.0, EPS, pos, turns, factor, rot, "half"
        want, bound = nu.norm_reference(*args)
        assert ((y.cpu().double() - want).abs() <= bound).all()
        for got, want, bound in zip((dx, dw), nu.gradients(*args, gy), nu.gradient_bounds(*args, gy)):
            assert ((got.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rot", [(64, 18), (96, 24), (128, 50), (256, 250)])
def test_new_tokens(dtype, d, rot):
    g = torch.Generator().manual_seed(d)
    T, Hq, Hkv, P, pages = 21, 5, 2, 16, 4
    q, k, v = (rows(g, T, h, d, dtype) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    slots = torch.randperm(P * pages, generator=g)[:T].to(torch.int32)
    slots[::4] = -1                                    # (rows of nobody between the others)
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0)
    ws = ws_of(g, d)
    kp, vp = (torch.full((pages, P, Hkv, d), 9.0, dtype=dtype, device=DEV) for _ in range(2))
    q_out = torch.full((T, Hq, d), 9.0, dtype=dtype, device=DEV)
    x = [t.to(DEV) for t in (q, k, v)]
    nb.stem_norm_rotary_append(db.RotaryShape.from_tensors(x[0], x[1], rot, "half", q_out), nb.HeadNorm(*(w.to(DEV) for w in ws), EPS, 0.0),
                               db.PageShape.from_tensors(kp, vp), *x, pos.to(DEV), slots.to(DEV), turns.to(DEV), factor, q_out, kp, vp)
    at = slots >= 0
    for t, w, y in ((q, ws[0], q_out.cpu()[at]), (k, ws[1], kp.cpu().view(-1, Hkv, d)[slots[at].long()])):
        want, bound = nu.norm_reference(t, w, 0.0, EPS, pos, turns, factor, rot, "half")
        assert ((y.double() - want[at]).abs() <= bound[at]).all()
    assert torch.equal(vp.cpu().view(-1, Hkv, d)[slots[at].long()], v[at])
    rest = torch.ones(P * pages, dtype=torch.bool)
    rest[slots[at].long()] = False
    assert (kp.cpu().view(-1, Hkv, d)[rest] == 9.0).all() and (vp.cpu().view(-1, Hkv, d)[rest] == 9.0).all()
    assert (q_out.cpu()[~at] == 9.0).all()


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 50), ("interleaved", 64)])
def test_long_calls(layout, rot):
    """Workgroups of several tokens, the last of them with fewer."""
    g = torch.Generator().manual_seed(rot)
    T, Hq, Hkv, d = 16387, 33, 4, 128
    q, k = (torch.randn(T, h, d, generator=g).to(BF) for h in (Hq, Hkv))
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0)
    ws = ws_of(g, d)
    x = [t.to(DEV) for t in (q, k)]
    out = [torch.full_like(t, float("nan")) for t in x]
    nb.stem_norm_rotary(db.RotaryShape.from_tensors(*x, rot, layout), nb.HeadNorm(*(w.to(DEV) for w in ws), EPS, 0.0), *x, pos.to(DEV),
                        turns.to(DEV), factor, *out)
    some = torch.cat([torch.arange(9), torch.arange(8000, 8009), torch.arange(T - 9, T)])
    for t, w, y in zip((q, k), ws, out):
        assert y.isfinite().all()
        want, bound = nu.norm_reference(t[some], w, 0.0, EPS, pos[some], turns, factor, rot, layout)
        assert ((y.cpu()[some].double() - want).abs() <= bound).all()
    # every row as in short calls
    for lo in range(0, T, 4000):
        part = [t[lo:lo + 4000] for t in x]
        again = [torch.empty_like(t) for t in part]
        nb.stem_norm_rotary(db.RotaryShape.from_tensors(*part, rot, layout), nb.HeadNorm(*(w.to(DEV) for w in ws), EPS, 0.0), *part,
                            pos[lo:lo + 4000].to(DEV), turns.to(DEV), factor, *again)
        for y, z in zip(out, again):
            assert torch.equal(y[lo:lo + 4000], z)


def test_norms_without_positions():
    from paper_2603_06274_amd.norm import NormRotary
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(40, h, 64, generator=g).to(BF) for h in (5, 2))
    ws = ws_of(g, 64)
    r = NormRotary.none(64, *(w.to(DEV) for w in ws), EPS)
    out = r.apply(q.to(DEV), k.to(DEV), torch.randint(0, 1 << 30, (40,), generator=g).to(torch.int32).to(DEV))
    for x, w, y in zip((q, k), ws, out):
        want, bound = nu.norm_reference(x, w, 0.0, EPS, torch.zeros(40, dtype=torch.int32), torch.zeros(1, dtype=torch.float64), 1.0, 2, "half")
        assert ((y.cpu().double() - want).abs() <= bound).all()
