"""stem_norm_rotary_append, and NormRotary in the place of Rotary: pre-filling, the paged cache, decoding steps."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import norm_binding as nb
from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode
from paper_2603_06274_amd.norm import NormRotary
from paper_2603_06274_amd.prefill import StemPrefill

import norm_util as nu
from test_gpu_norm_rotary import BF, DEV, EPS, FP, HF, check, make, on_gpu, places, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,page", [(1, 8, 2, 128, 128, 16), (70, 28, 4, 128, 64, 64), (9, 0, 3, 64, 20, 32),
                                                 (33, 4, 1, 256, 256, 128), (300, 2, 2, 24, 16, 256), (5, 1, 1, 1024, 1000, 16)])
def test_append(dtype, layout, T, Hq, Hkv, d, rot, page):
    """Rows that have a place, in the order of no other; those without one are left alone, and so is the rest of the pages."""
    q, k, v = make(T, Hq, Hkv, d, dtype, seed=T, packed=True)
    q = q if Hq else None
    turns, factor = db.stem_rotary_frequencies(rot, 500000.0)
    pos, ws = places(T), weights_of(d, dtype, 0.0)
    pages = -(-T // page) + 2
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    if T > 4:
        slots[1], slots[3] = -1, pages * page
    kp, vp = (torch.full((pages, page, Hkv, d), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    q_out = None if q is None else torch.full((T, Hq, d), 7.0, dtype=dtype, device=DEV)
    shape, norm = db.RotaryShape.from_tensors(q, k, rot, layout, q_out), nb.HeadNorm(*on_gpu(ws), EPS)
    nb.stem_norm_rotary_append(shape, norm, db.PageShape.from_tensors(kp, vp), q, k, v, pos.to(DEV), slots.to(DEV), turns.to(DEV), factor,
                               q_out, kp, vp)
    there = ((slots >= 0) & (slots < pages * page)).nonzero()[:, 0]
    if q is not None:
        want, bound = nu.norm_reference(q.cpu(), ws[0], 0.0, EPS, pos, turns, factor, rot, layout)
        check(q_out[there], want[there], bound[there], "q")
        rest = torch.ones(T, dtype=torch.bool)
        rest[there] = False
        assert (q_out[rest] == 7.0).all()
    want, bound = nu.norm_reference(k.cpu(), ws[1], 0.0, EPS, pos, turns, factor, rot, layout)
    flat_k, flat_v = kp.view(-1, Hkv, d), vp.view(-1, Hkv, d)
    at = slots[there].long().to(DEV)
    check(flat_k[at], want[there], bound[there], "k")
    assert torch.equal(flat_v[at], v[there.to(DEV)])
    flat_k[at], flat_v[at] = 7.0, 7.0
    assert (kp == 7.0).all() and (vp == 7.0).all()


def test_takes_the_place_of_rotary():
    """Pre-filling and steps with NormRotary are those with Rotary of rows that were normalised before (without positions, so that both
    round once to the same value)."""
    T, Hq, Hkv, d, R = 700, 4, 2, 128, 3
    q, k, v = make(T, Hq, Hkv, d, BF)
    ws = on_gpu(weights_of(d, BF, 0.0))
    norm = NormRotary.none(d, *ws, EPS)
    before = norm.apply(q, k, torch.zeros(T, dtype=torch.int32, device=DEV))
    steps = [make(R, Hq, Hkv, d, BF, seed=50 + i) for i in range(3)]

    def go(rotary, q, k, steps):
        pf = StemPrefill(q, k, v, [0, T], 64, [4], rotary=rotary)
        outs = [pf.run().clone()]
        decode = pf.decode(PagedCache(R, 9, 16, 3, Hkv, d))
        for x in steps:
            outs.append(decode.step(*x).clone())
        return outs

    none = torch.zeros(R, dtype=torch.int32, device=DEV)
    turned = [(*norm.apply(a, b, none), c) for a, b, c in steps]
    for x, y in zip(go(norm, q, k, steps), go(Rotary.none(d), *before, turned)):
        assert torch.equal(x, y)


def test_a_step_with_unfit_weights_leaves_the_cache():
    d, R = 64, 2
    cache = PagedCache(R, 8, 16, 4, 1, d)
    prefix = torch.randn(40, 1, d, device=DEV).to(BF)
    decode = StemDecode(prefix, prefix, 2, cache, NormRotary(d, None, torch.ones(d, device=DEV), EPS))
    rows = make(R, 2, 1, d, BF)
    decode.rotary.norm.k_weight = torch.ones(d + 8, device=DEV)
    with pytest.raises(ValueError):
        decode.step(*rows)
    torch.cuda.synchronize()
    assert cache.lens.tolist() == [0, 0] and cache.ring_state.tolist() == [0, 8]
