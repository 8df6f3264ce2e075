"""stem_rotary_append: what goes to the pages, what is left alone, strides, slots that are none, caches beyond 32 bits."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db

import decode_util as du
from test_gpu_rotary import BF, DEV, FP, HF, check, make

pytestmark = pytest.mark.gpu


def run(q, k, v, pos, slots, turns, factor, rot, layout, q_out, kp, vp):
    shape = db.RotaryShape.from_tensors(q, k, rot, layout, q_out)
    db.stem_rotary_append(shape, db.PageShape.from_tensors(kp, vp), q, k, v, pos.to(DEV), slots.to(DEV), turns.to(DEV), factor, q_out,
                          kp, vp)


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,P,heads_first", [
    (1, 32, 8, 128, 128, 16, False), (64, 8, 2, 64, 32, 64, True), (77, 28, 4, 128, 128, 16, True), (300, 0, 2, 256, 64, 32, False),
    (1200, 2, 1, 64, 20, 128, False), (4500, 1, 1, 64, 64, 256, True)])
def test_append(dtype, layout, T, Hq, Hkv, d, rot, P, heads_first):
    q, k, v = make(T, Hq, Hkv, d, dtype, seed=T, packed=T == 77)
    q = q if Hq else None
    turns, factor = db.stem_rotary_frequencies(rot, 10000.0, "yarn", 4.0, 4096.0, 1.0, 32.0)
    g = torch.Generator().manual_seed(3)
    N = -(-T // P) + 2
    pos = torch.randint(0, 1 << 18, (T,), generator=g).to(torch.int32)
    slots = torch.randperm(N * P, generator=g)[:T].to(torch.int32)
    none = torch.rand(T, generator=g) < 0.2 if T > 1 else torch.zeros(T, dtype=torch.bool)
    slots[none] = torch.tensor([-1, N * P, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).repeat(T)[:int(none.sum())]
    if heads_first:
        kp, vp = (torch.full((N, Hkv, P, d), 3.0, dtype=dtype, device=DEV).transpose(1, 2) for _ in range(2))
    else:
        kp, vp = (torch.full((N, P, Hkv, d), 3.0, dtype=dtype, device=DEV) for _ in range(2))
    q_out = torch.full((T, Hq, d), 5.0, dtype=dtype, device=DEV) if Hq else None
    run(q, k, v, pos, slots, turns, factor, rot, layout, q_out, kp, vp)
    there = (~none).nonzero()[:, 0]
    if Hq:
        want, bound = du.rotary_reference(q.cpu(), pos, turns, factor, rot, layout)
        check(q_out.cpu()[there], want[there], bound[there], "q")
        assert (q_out.cpu()[none] == 5.0).all()
    want, bound = du.rotary_reference(k.cpu(), pos, turns, factor, rot, layout)
    at = slots.long()[there]
    got_k, got_v = kp.cpu(), vp.cpu()
    check(got_k[at // P, at % P], want[there], bound[there], "k")
    assert torch.equal(got_v[at // P, at % P], v.cpu()[there])
    got_k[at // P, at % P], got_v[at // P, at % P] = 3.0, 3.0
    assert (got_k == 3.0).all() and (got_v == 3.0).all()


def test_the_same_as_rotary():
    """The same bits as stem_rotary's."""
    q, k, v = make(50, 4, 2, 128, BF)
    turns, factor = db.stem_rotary_frequencies(128, 10000.0)
    pos = torch.arange(50, dtype=torch.int32) * 99
    kp, vp = (torch.zeros(4, 16, 2, 128, dtype=BF, device=DEV) for _ in range(2))
    q_out, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
    run(q, k, v, pos, torch.arange(50, dtype=torch.int32), turns, factor, 128, "half", q_out, kp, vp)
    db.stem_rotary(db.RotaryShape.from_tensors(q, k, 128), q, k, pos.to(DEV), turns.to(DEV), factor, q2, k2)
    assert torch.equal(q_out, q2) and torch.equal(kp.view(64, 2, 128)[:50], k2) and torch.equal(vp.view(64, 2, 128)[:50], v)


def test_values_that_are_not_finite_go_to_the_pages_as_they_are():
    q, k, v = make(4, 1, 1, 64, BF)
    v[0, 0, 3], v[1, 0, 40], v[2, 0, 5] = float("inf"), float("nan"), float("-inf")
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    for layout in ("half", "interleaved"):
        kp, vp = (torch.zeros(1, 16, 1, 64, dtype=BF, device=DEV) for _ in range(2))
        run(q, k, v, torch.arange(4, dtype=torch.int32), torch.arange(4, dtype=torch.int32), turns, factor, 64, layout,
            torch.empty_like(q), kp, vp)
        assert torch.equal(vp[0, :4].view(torch.int16), v.view(torch.int16))


def test_a_cache_beyond_32_bits():
    """Pages whose elements lie beyond 2^32: 5 GB of bf16 with a wide stride between pages."""
    N, P, H, d = 9, 16, 1, 64
    room = torch.zeros(N, 300_000_000, dtype=BF, device=DEV)
    kp = room[:, :P * H * d].unflatten(1, (P, H, d))
    vp = room[:, 4096:4096 + P * H * d].unflatten(1, (P, H, d))
    q, k, v = make(3, 2, 1, 64, BF)
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    pos, slots = torch.tensor([7, 8, 9], dtype=torch.int32), torch.tensor([8 * 16 + 15, 7 * 16, 0], dtype=torch.int32)
    q_out = torch.empty_like(q)
    run(q, k, v, pos, slots, turns, factor, 64, "half", q_out, kp, vp)
    want, bound = du.rotary_reference(k.cpu(), pos, turns, factor, 64, "half")
    got = torch.stack([kp[8, 15], kp[7, 0], kp[0, 0]])
    check(got, want, bound, "k")
    assert torch.equal(torch.stack([vp[8, 15], vp[7, 0], vp[0, 0]]), v)
    assert int((kp != 0).sum()) <= 3 * 64 and int((room[8] != 0).sum()) <= 2 * 64
