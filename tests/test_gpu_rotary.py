"""stem_rotary against its formula in 64 bits: types, layouts, parts of the head, sizes, strides, in place, the transposed map."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db

import decode_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def make(T, Hq, Hkv, d, dtype, seed=0, packed=False):
    g = torch.Generator().manual_seed(seed)
    if packed:                                         # one tensor [T, Hq + 2 Hkv, d] as a projection leaves it
        x = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(dtype).to(DEV)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return tuple(torch.randn(T, h, d, generator=g).to(dtype).to(DEV) for h in (Hq, Hkv, Hkv))


def check(got, want, bound, what):
    off = (got.cpu().double() - want).abs()
    assert (off <= bound).all(), "%s: %g over, worst %g" % (what, (off - bound).max(), off.max())


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,packed", [
    (1, 32, 8, 128, 128, False), (1, 1, 1, 8, 2, False), (7, 28, 4, 128, 64, True), (300, 4, 2, 64, 64, True),
    (33, 5, 0, 256, 96, False), (33, 0, 3, 64, 20, False), (5, 3, 3, 72, 72, False), (1500, 2, 1, 64, 48, False),
    (4100, 2, 1, 64, 64, False), (4097, 1, 1, 32, 10, True), (3, 2, 1, 1024, 1024, False), (4099, 1, 1, 1024, 1000, False)])
def test_rotary_matches_its_formula(dtype, layout, T, Hq, Hkv, d, rot, packed):
    q, k, _ = make(T, Hq, Hkv, d, dtype, seed=T + d, packed=packed)
    q, k = (q if Hq else None), (k if Hkv else None)
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0, "yarn", 8.0, 8192.0, 1.0, 32.0)
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    pos[0] = -5 if T > 1 else 131071
    pos[-1] = (1 << 31) - 1 if T > 2 else pos[-1]
    for backward in (False, True):
        outs = [torch.full_like(x, float("nan")) if x is not None else None for x in (q, k)]
        shape = db.RotaryShape.from_tensors(q, k, rot, layout, *outs)
        db.stem_rotary(shape, q, k, pos.to(DEV), turns.to(DEV), factor, *outs, backward)
        for name, x, y in zip("qk", (q, k), outs):
            if x is not None:
                want, bound = du.rotary_reference(x.cpu(), pos, turns, factor, rot, layout, backward)
                check(y, want, bound, (name, backward))
        # in place: the same bits
        copies = [x.clone() if x is not None else None for x in (q, k)]
        shape = db.RotaryShape.from_tensors(*copies, rot, layout)
        db.stem_rotary(shape, *copies, pos.to(DEV), turns.to(DEV), factor, *copies, backward)
        for x, y in zip(copies, outs):
            assert x is None or torch.equal(x, y.reshape(x.shape))


def test_rows_behind_the_call_and_between_heads_stay():
    """Outputs with gaps: heads in a wider row, tokens of a longer tensor."""
    q, k, _ = make(9, 3, 1, 64, BF)
    wide = torch.full((12, 8, 96), 7.0, dtype=BF, device=DEV)
    q_out, k_out = wide[:9, :3, :64], wide[:9, 4:5, 8:72]
    turns, factor = db.stem_rotary_frequencies(32, 10000.0)
    pos = torch.arange(20, dtype=torch.int32)
    db.stem_rotary(db.RotaryShape.from_tensors(q, k, 32, "half", q_out, k_out), q, k, pos.to(DEV), turns.to(DEV), factor, q_out, k_out)
    want, bound = du.rotary_reference(q.cpu(), pos[:9], turns, factor, 32, "half")
    check(q_out, want, bound, "q")
    want, bound = du.rotary_reference(k.cpu(), pos[:9], turns, factor, 32, "half")
    check(k_out, want, bound, "k")
    q_out.fill_(7.0), k_out.fill_(7.0)
    assert (wide == 7.0).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_backward_is_the_gradient(layout):
    """In fp32: <g, R(x + u) - R(x - u)> / 2 = <R^T g, u>, and the gradients that autograd finds of the formula."""
    T, H, d, rot = 40, 3, 64, 48
    g = torch.Generator().manual_seed(4)
    x, u, gr = (torch.randn(T, H, d, generator=g) for _ in range(3))
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0, "yarn", 4.0, 2048.0, 1.0, 32.0)
    pos = torch.randint(0, 100000, (T,), generator=g).to(torch.int32)
    shape = db.RotaryShape.from_tensors(x.to(DEV), None, rot, layout)

    def run(v, backward):
        v = v.to(DEV)
        y = torch.empty_like(v)
        db.stem_rotary(shape, v, None, pos.to(DEV), turns.to(DEV), factor, y, None, backward)
        return y.cpu().double()

    back = run(gr, True)
    x64 = x.double().requires_grad_()
    du.rotary_reference(x64, pos, turns, factor, rot, layout)[0].backward(gr.double())
    _, bound = du.rotary_reference(gr, pos, turns, factor, rot, layout, True)
    assert ((back - x64.grad).abs() <= bound).all()
    difference = ((run(x + u, False) - run(x - u, False)) / 2 * gr.double()).sum()
    # each of the T H d terms: 10 u (|x1| + |x2|) f of either side, and the sums x + u, x - u round: 2^-24 of at most 6
    assert abs(difference - (back * u.double()).sum()) <= T * H * d * 12 * du.U * factor * 8 * 4


def test_replays_follow_the_positions():
    q, k, _ = make(6, 4, 2, 64, BF)
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    pos, td = torch.zeros(6, dtype=torch.int32, device=DEV), turns.to(DEV)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    shape = db.RotaryShape.from_tensors(q, k, 64, "half", q_out, k_out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        db.stem_rotary(shape, q, k, pos, td, factor, q_out, k_out)
    for step in range(4):
        pos.copy_(torch.arange(6, dtype=torch.int32) + 1000 * step)
        q_out.zero_(), k_out.zero_()
        graph.replay()
        eager = torch.empty_like(q), torch.empty_like(k)
        db.stem_rotary(shape, q, k, pos, td, factor, *eager)
        torch.cuda.synchronize()
        assert torch.equal(q_out, eager[0]) and torch.equal(k_out, eager[1])


def test_runs_on_the_current_stream():
    q, k, _ = make(2000, 8, 2, 128, BF)
    turns, factor = db.stem_rotary_frequencies(128, 10000.0)
    pos, td = torch.arange(2000, dtype=torch.int32, device=DEV), turns.to(DEV)
    shape = db.RotaryShape.from_tensors(q, k, 128)
    want = torch.empty_like(q), torch.empty_like(k)
    db.stem_rotary(shape, q, k, pos, td, factor, *want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = torch.empty_like(q), torch.empty_like(k)
    with torch.cuda.stream(side):
        later = q * 1.0                                # on the side stream, before the call
        db.stem_rotary(shape, later, k, pos, td, factor, *got)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
