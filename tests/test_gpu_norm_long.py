"""Calls of normalised heads as long as a training step's or a busy server's: gradients whose sums are over hundreds of workgroups, values
past the caches, and new rows past them."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import norm_binding as nb

import norm_util as nu
from test_gpu_norm_rotary import BF, DEV, EPS, FP, HF, check, on_gpu, weights_of

pytestmark = pytest.mark.gpu


def rows(g, T, H, d, dtype):
    return torch.randn(T, H, d, generator=g, device=DEV).to(dtype)


def parts(T, H, d):
    """Workgroups of the backward pass, each with a sum, by the size of their workspace (2 sums of d fp32 values each)."""
    x = torch.empty(T, H, d, device="meta", dtype=BF)
    return nb.stem_norm_rotary_backward_workspace_bytes(db.RotaryShape.from_tensors(x, None, d)) // (8 * d)


@pytest.mark.parametrize("dtype,layout,T,Hq,Hkv,d,rot", [
    (BF, "half", 2050, 16, 4, 128, 128),               # 512 sums
    (FP, "interleaved", 9001, 5, 2, 64, 64),           # 393
    (HF, "half", 4099, 9, 2, 128, 50),                 # 563, halves inside chunks
    (BF, "half", 16387, 33, 4, 128, 128),              # 1024 sums, 155 MB of values: past the caches
    (BF, "half", 16387, 33, 4, 128, 50),
    (HF, "interleaved", 16387, 33, 4, 128, 64),
    (FP, "half", 16387, 9, 1, 128, 126),
    (FP, "half", 9001, 3, 1, 1024, 1000)])             # one wave per head
def test_gradients(dtype, layout, T, Hq, Hkv, d, rot):
    """All sums, and rows at the calls' ends and between."""
    g = torch.Generator(device=DEV).manual_seed(T + rot)
    q, k, gq, gk = (rows(g, T, h, d, dtype) for h in (Hq, Hkv, Hq, Hkv))
    assert parts(T, Hq + Hkv, d) > 256
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, device=DEV).to(torch.int32)
    ws = on_gpu(weights_of(d, dtype, 0.0))
    shape = db.RotaryShape.from_tensors(q, k, rot, layout)
    space = torch.full((nb.stem_norm_rotary_backward_workspace_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    grads, sums = [torch.full_like(x, float("nan")) for x in (q, k)], [torch.full((d,), float("nan"), device=DEV) for _ in ws]
    nb.stem_norm_rotary_backward(shape, nb.HeadNorm(*ws, EPS), q, k, pos, turns.to(DEV), factor, gq, gk, *grads, *sums, space)
    some = torch.cat([torch.arange(9), torch.arange(T // 2, T // 2 + 9), torch.arange(T - 9, T)]).to(DEV)
    for x, gy, w, dx, dw in zip((q, k), (gq, gk), ws, grads, sums):
        assert dx.isfinite().all()
        args = x[some].cpu(), w.cpu(), 0.0, EPS, pos[some].cpu(), turns, factor, rot, layout, gy[some].cpu()
        check(dx[some], nu.gradients(*args)[0], nu.gradient_bounds(*args)[0], "dx")
        want, bound = torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
        # (on the GPU, in 64 bits, a few rows at a time; a bound of terms adds up as they do, but for the number of sums in a row, which is T's)
        for lo in range(0, T, 4096):
            at = slice(lo, lo + 4096)
            args = x[at], w, 0.0, EPS, pos[at], turns.to(DEV), factor, rot, layout, gy[at]
            want += nu.gradients(*args)[1].cpu()
            bound += nu.gradient_bounds(*args)[1].cpu() * -(-T // 4096)
        check(dw, want, bound, "dw")
    # the same bits for the same inputs, and in place of the outputs' gradients
    again = [torch.empty_like(x) for x in sums]
    nb.stem_norm_rotary_backward(shape, nb.HeadNorm(*ws, EPS), q, k, pos, turns.to(DEV), factor, gq, gk, gq, gk, *again, space)
    for x, y in zip((gq, gk, *again), (*grads, *sums)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 50), ("interleaved", 64)])
def test_new_rows(layout, rot):
    """More than the caches hold, some without a place: as in calls of few rows, and the rest of the pages as it was."""
    T, Hq, Hkv, d, P = 9001, 32, 4, 128, 16
    g = torch.Generator(device=DEV).manual_seed(rot)
    q, k, v = (rows(g, T, h, d, BF) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 1 << 20, (T,), generator=g, device=DEV).to(torch.int32)
    pages = T // P + 9
    slots = torch.randperm(pages * P, generator=g, device=DEV)[:T].to(torch.int32)
    slots[::7] = -1
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0)
    ws = weights_of(d, BF, 0.0)
    norm = nb.HeadNorm(*on_gpu(ws), EPS)

    def go(step):
        kp, vp = (torch.full((pages, P, Hkv, d), 7.0, dtype=BF, device=DEV) for _ in range(2))
        q_out = torch.full_like(q, 7.0)
        for lo in range(0, T, step):
            at = slice(lo, lo + step)
            shape = db.RotaryShape.from_tensors(q[at], k[at], rot, layout, q_out[at])
            nb.stem_norm_rotary_append(shape, norm, db.PageShape.from_tensors(kp, vp), q[at], k[at], v[at], pos[at], slots[at], turns.to(DEV),
                                       factor, q_out[at], kp, vp)
        return q_out, kp, vp

    one, many = go(T), go(500)
    for x, y in zip(one, many):
        assert torch.equal(x, y)
    there = slots >= 0
    assert (one[0][~there] == 7.0).all() and torch.equal(one[2].view(-1, Hkv, d)[slots[there].long()], v[there])
    some = there.nonzero()[:, 0][::500]
    for x, w, y in ((q, ws[0], one[0][some]), (k, ws[1], one[1].view(-1, Hkv, d)[slots[some].long()])):
        want, bound = nu.norm_reference(x[some].cpu(), w, 0.0, EPS, pos[some].cpu(), turns, factor, rot, layout)
        check(y, want, bound, "row")
