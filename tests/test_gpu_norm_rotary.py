"""stem_norm_rotary and its gradients against their formulas in 64 bits: types, layouts, parts of the head, weights, sizes, strides, in
place; non-finite heads; captured calls; autograd through NormRotary."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import norm_binding as nb
from paper_2603_06274_amd.norm import NormRotary

import norm_util as nu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
EPS = 2.0 ** -20                                       # a number of fp32


def make(T, Hq, Hkv, d, dtype, seed=0, packed=False):
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(torch.randn(Hq + 2 * Hkv, 1, generator=g))
    x = (torch.randn(T, Hq + 2 * Hkv, d, generator=g) * size).to(dtype).to(DEV)
    parts = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return parts if packed else tuple(p.contiguous() for p in parts)


def weights_of(d, kind, offset, seed=3):
    g = torch.Generator().manual_seed(seed)
    return [None if kind is None else (1.0 - offset + 0.3 * torch.randn(d, generator=g)).to(kind) for _ in range(2)]


def on_gpu(ws):
    return [w if w is None else w.to(DEV) for w in ws]


def check(got, want, bound, what):
    off = (got.cpu().double() - want).abs()
    assert (off <= bound).all(), "%s: %g over, worst %g" % (what, (off - bound).max(), off.max())


def places(T, seed=1):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    pos[0] = -5 if T > 1 else 131071
    if T > 2:
        pos[-1] = (1 << 31) - 1
    return pos


SIZES = [(1, 32, 8, 128, 128, False), (1, 1, 1, 8, 2, False), (7, 28, 4, 128, 64, True), (300, 4, 2, 64, 64, True),
         (33, 5, 0, 256, 96, False), (33, 0, 3, 64, 20, False), (5, 3, 3, 72, 72, False), (9, 2, 2, 24, 16, False), (9, 2, 1, 104, 32, True),
         (1500, 2, 1, 64, 48, False), (4100, 2, 1, 64, 64, False), (4097, 1, 1, 32, 10, True), (3, 2, 1, 1024, 1024, False),
         (130, 1, 1, 1024, 1000, False), (20, 3, 2, 512, 256, False), (64, 40, 1, 128, 128, False)]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,packed", SIZES)
def test_matches_its_formula(dtype, layout, T, Hq, Hkv, d, rot, packed):
    q, k, _ = make(T, Hq, Hkv, d, dtype, seed=T + d, packed=packed)
    q, k = (q if Hq else None), (k if Hkv else None)
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0, "yarn", 8.0, 8192.0, 1.0, 32.0)
    pos = places(T)
    kind, offset = [(dtype, 0.0), (FP, 1.0), (None, 0.0)][(T + d // 8) % 3]
    ws = weights_of(d, kind, offset)
    norm = nb.HeadNorm(*on_gpu(ws), EPS, offset)
    outs = [torch.full_like(x, float("nan")) if x is not None else None for x in (q, k)]
    shape = db.RotaryShape.from_tensors(q, k, rot, layout, *outs)
    nb.stem_norm_rotary(shape, norm, q, k, pos.to(DEV), turns.to(DEV), factor, *outs)
    for name, x, y, w in zip("qk", (q, k), outs, ws):
        if x is not None:
            check(y, *nu.norm_reference(x.cpu(), w, offset, EPS, pos, turns, factor, rot, layout), name)
    copies = [x.clone() if x is not None else None for x in (q, k)]                # in place: the same bits
    shape = db.RotaryShape.from_tensors(*copies, rot, layout)
    nb.stem_norm_rotary(shape, norm, *copies, pos.to(DEV), turns.to(DEV), factor, *copies)
    for x, y in zip(copies, outs):
        assert x is None or torch.equal(x, y)


def backward_call(q, k, gq, gk, rot, layout, norm, pos, turns, factor, dq, dk, sums):
    shape = db.RotaryShape.from_tensors(q, k, rot, layout, gq, gk)
    space = torch.full((nb.stem_norm_rotary_backward_workspace_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    nb.stem_norm_rotary_backward(shape, norm, q, k, pos.to(DEV), turns.to(DEV), factor, gq, gk, dq, dk, *sums, space)


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,packed", SIZES)
def test_gradients_match_their_formula(dtype, layout, T, Hq, Hkv, d, rot, packed):
    q, k, _ = make(T, Hq, Hkv, d, dtype, seed=T + d, packed=packed)
    q, k = (q if Hq else None), (k if Hkv else None)
    g = torch.Generator().manual_seed(9)
    gq, gk = (torch.randn(T, h, d, generator=g).to(dtype).to(DEV) if h else None for h in (Hq, Hkv))
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0, "yarn", 8.0, 8192.0, 1.0, 32.0)
    pos = places(T)
    kind, offset = [(dtype, 0.0), (FP, 1.0), (None, 0.0)][(T + d // 8 + 1) % 3]
    ws = weights_of(d, kind, offset)
    norm = nb.HeadNorm(*on_gpu(ws), EPS, offset)
    grads = [torch.empty_strided(x.shape, x.stride(), dtype=dtype, device=DEV) if x is not None else None for x in (q, k)]
    sums = [None if w is None else torch.full((d,), float("nan"), device=DEV) for w in ws]
    backward_call(q, k, gq, gk, rot, layout, norm, pos, turns, factor, *grads, sums)
    for name, x, gy, dx, w, dw in zip("qk", (q, k), (gq, gk), grads, ws, sums):
        if x is None:
            assert dw is None or (dw == 0).all()
            continue
        args = x.cpu(), w, offset, EPS, pos, turns, factor, rot, layout, gy.cpu()
        (want, want_w), (bound, bound_w) = nu.gradients(*args), nu.gradient_bounds(*args)
        check(dx, want, bound, name)
        if w is not None:
            check(dw, want_w, bound_w, name + " weight")
    # once more, over the inputs where strides allow it: the same bits
    places_of = [x.clone() if x is not None else None for x in (gq, gk)]
    again = [None if w is None else torch.empty(d, device=DEV) for w in ws]
    if all(x is None or x.stride() == y.stride() for x, y in zip((q, k), places_of)):
        backward_call(q, k, *places_of, rot, layout, norm, pos, turns, factor, *places_of, again)
        for x, y in zip(places_of, grads):
            assert x is None or torch.equal(x, y)
        for x, y in zip(again, sums):
            assert x is None or torch.equal(x, y)


@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 40), ("half", 20)])
def test_the_formula_of_the_gradients_by_differences(layout, rot):
    """In 64 bits, on the CPU: <dx, a> + <dw, b> is the derivative along (a, b), by central differences at two steps whose errors of the
    second order cancel; what is left is of the fourth order (10^-3 to the fourth, times derivatives of the order of 10^3) and 2^-52 / 10^-3
    of the sums."""
    T, H, d = 6, 2, 64
    g = torch.Generator().manual_seed(5)
    x, a, gy = (torch.randn(T, H, d, generator=g, dtype=torch.float64) for _ in range(3))
    w, b = 1 + 0.2 * torch.randn(d, generator=g, dtype=torch.float64), torch.randn(d, generator=g, dtype=torch.float64)
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0)
    pos = torch.arange(T, dtype=torch.int32) * 1000

    def loss(t):
        return (nu.turned(nu.normed(x + t * a, w + t * b, 0.5, 1e-6), pos, turns, factor, rot, layout) * gy).sum()

    dx, dw = nu.gradients(x, w, 0.5, 1e-6, pos, turns, factor, rot, layout, gy)
    h = 1e-3
    one, two = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
    assert ((4 * one - two) / 3 - (dx * a).sum() - (dw * b).sum()).abs() <= 1e-8
    # and the kernel's derivative along a, in fp32, is that of the formula
    dxk, dwk = torch.empty(T, H, d, device=DEV), torch.empty(d, device=DEV)
    norm = nb.HeadNorm(w.float().to(DEV), None, 1e-6, 0.5)
    xf, wf, gf = x.float(), w.float(), gy.float()
    shape = db.RotaryShape.from_tensors(xf.to(DEV), None, rot, layout)
    space = torch.empty(nb.stem_norm_rotary_backward_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    nb.stem_norm_rotary_backward(shape, norm, xf.to(DEV), None, pos.to(DEV), turns.to(DEV), factor, gf.to(DEV), None, dxk, None, dwk, None,
                                 space)
    args = xf, wf, 0.5, nb._f32(1e-6).value, pos, turns, factor, rot, layout, gf
    (want, want_w), (bound, bound_w) = nu.gradients(*args), nu.gradient_bounds(*args)
    check(dxk, want, bound, "dx")
    check(dwk, want_w, bound_w, "dw")


def test_rows_of_zeros_and_small_values():
    """A head of zeros gives zeros, and values whose squares vanish beside eps are divided by its root."""
    x = torch.zeros(3, 2, 64, device=DEV)
    x[1] = 1e-18
    x[2, 1] = 1e15
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    pos = torch.zeros(3, dtype=torch.int32)
    out = torch.empty_like(x)
    nb.stem_norm_rotary(db.RotaryShape.from_tensors(x, None, 64), nb.HeadNorm(None, None, EPS), x, None, pos.to(DEV), turns.to(DEV), factor,
                        out, None)
    check(out, *nu.norm_reference(x.cpu(), None, 0.0, EPS, pos, turns, factor, 64, "half"), "y")
    assert (out[0] == 0).all()


@pytest.mark.parametrize("rot", [64, 20])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_head_that_is_not_finite_stays_by_itself(rot, value):
    """Every other head's values and gradients keep their bits."""
    q, k, _ = make(40, 6, 2, 64, BF)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0)
    pos = torch.arange(40, dtype=torch.int32)
    norm = nb.HeadNorm(None, None, EPS)

    def both():
        outs, grads = [torch.empty_like(x) for x in (q, k)], [torch.empty_like(x) for x in (q, k)]
        nb.stem_norm_rotary(db.RotaryShape.from_tensors(q, k, rot), norm, q, k, pos.to(DEV), turns.to(DEV), factor, *outs)
        backward_call(q, k, gq, gk, rot, "half", norm, pos, turns, factor, *grads, (None, None))
        return outs[0], grads[0], outs[1], grads[1]

    then = both()
    q[7, 3, 5] = value
    now = both()
    for x, y in zip(then[:2], now[:2]):
        same = torch.ones(40, 6, dtype=torch.bool, device=DEV)
        same[7, 3] = False
        assert torch.equal(x[same], y[same]) and not torch.equal(x[7, 3], y[7, 3])
    assert torch.equal(then[2], now[2]) and torch.equal(then[3], now[3])


def test_no_tokens():
    """Weights' gradients of no tokens are 0."""
    x = torch.empty(0, 2, 64, device=DEV)
    norm = nb.HeadNorm(torch.ones(64, device=DEV), None, EPS)
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    dw = torch.full((64,), 7.0, device=DEV)
    backward_call(x, None, x, None, 64, "half", norm, torch.zeros(0, dtype=torch.int32), turns, factor, x, None, (dw, None))
    assert (dw == 0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_autograd(dtype):
    """NormRotary carries the gradients of rows and weights, also where one part has none, or a gradient comes without strides."""
    T, Hq, Hkv, d = 50, 4, 2, 64
    rows = make(T, Hq, Hkv, d, dtype, packed=True)
    ws = [w.to(DEV).requires_grad_() for w in weights_of(d, dtype, 0.0)]
    rotary = NormRotary(d, *ws, EPS, theta=10000.0)
    pos = torch.arange(T, dtype=torch.int32)
    q, k = (x.detach().clone().requires_grad_() for x in rows[:2])
    gy = torch.randn(T, Hq, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    out_q, out_k = rotary.apply(q, k, pos.to(DEV))
    ((out_q * gy.to(DEV)).sum() + 2.0 * out_k.sum()).backward()
    for x, w, g in ((q, ws[0], gy), (k, ws[1], torch.full((T, Hkv, d), 2.0, dtype=dtype))):
        args = x.detach().cpu(), w.detach().cpu(), 0.0, EPS, pos, rotary.turns.cpu(), 1.0, d, "half", g
        (want, want_w), (bound, bound_w) = nu.gradients(*args), nu.gradient_bounds(*args)
        check(x.grad, want, bound, "x")
        check(w.grad, want_w, bound_w + nu.EPS[dtype] / 2 * (want_w.abs() + bound_w), "w")
    for t in (q, k, *ws):
        t.grad = None
    out_q, out_k = rotary.apply(q, k, pos.to(DEV))     # keys alone have something to say
    out_k.sum().backward()
    assert q.grad is None and ws[0].grad is None and k.grad is not None and ws[1].grad is not None
    k.grad = None
    rotary.apply(None, k, pos.to(DEV))[1].sum().backward()
    assert k.grad is not None
    plain_q, plain_k = rotary.apply(q.detach(), k, pos.to(DEV))
    assert plain_q.requires_grad and plain_k.requires_grad                       # (the weights' gradients)
    with torch.no_grad():
        assert not rotary.apply(q, k, pos.to(DEV))[0].requires_grad
    with pytest.raises(ValueError, match="carry no gradients"):
        rotary.apply(q, k, pos.to(DEV), torch.empty_like(q), torch.empty_like(k))
    with pytest.raises(TypeError):
        rotary.backward(q, k, pos.to(DEV))


def test_gradients_method_and_shared_weights():
    """One weight for queries and keys gets the sum of both gradients from autograd; gradients() gives them apart."""
    T, d = 30, 128
    q, k, _ = make(T, 4, 1, d, FP)
    w = weights_of(d, FP, 0.0)[0].to(DEV).requires_grad_()
    rotary = NormRotary(d, w, w, EPS)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    dq, dk, dqw, dkw = rotary.gradients(q, k, gq, gk, pos)
    q.requires_grad_(), k.requires_grad_()
    torch.autograd.backward(rotary.apply(q, k, pos), (gq, gk))
    assert torch.equal(q.grad, dq) and torch.equal(k.grad, dk) and torch.equal(w.grad, dqw + dkw)


def test_captured():
    """Both directions in a graph, replayed with other inputs and eager work between; the same bits as eager calls."""
    T, d = 700, 128
    q, k, _ = make(T, 8, 2, d, BF)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    ws = on_gpu(weights_of(d, BF, 0.0))
    norm = nb.HeadNorm(*ws, EPS)
    turns, factor = db.stem_rotary_frequencies(d, 10000.0)
    turns, pos = turns.to(DEV), torch.arange(T, dtype=torch.int32, device=DEV)
    shape = db.RotaryShape.from_tensors(q, k, d)
    space = torch.empty(nb.stem_norm_rotary_backward_workspace_bytes(shape), dtype=torch.uint8, device=DEV)

    def run(into):
        nb.stem_norm_rotary(shape, norm, q, k, pos, turns, factor, into[0], into[1])
        nb.stem_norm_rotary_backward(shape, norm, q, k, pos, turns, factor, gq, gk, into[2], into[3], into[4], into[5], space)

    def buffers():
        return [torch.zeros_like(x) for x in (q, k, q, k)] + [torch.zeros(d, device=DEV) for _ in range(2)]

    captured, eager = buffers(), buffers()
    run(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(captured)
    for turn in range(4):
        q.copy_(torch.randn_like(q)), gq.copy_(torch.randn_like(gq)), ws[0].mul_(1.1)
        run(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured, eager):
            assert torch.equal(x, y)
