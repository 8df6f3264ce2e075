"""Values of new tokens that are not finite, where their weight is next to nothing: they reach the rows that see them all the same, an
infinite one as itself, in one launch and in two, whichever waves or parts have met the rows' other keys."""
import math

import pytest
import torch

from test_gpu_prefix_attn import BF, HF
from test_gpu_tree_attn import TreeCase
from test_gpu_tree_attn_launches import with_room

pytestmark = pytest.mark.gpu


def check(c, j, value):
    """Value 5 of KV head 1 of request 0's new token j becomes `value`: so do the outputs of the rows that see it, and nothing else changes."""
    clean, z = c.run()
    assert clean.isfinite().all()
    page, at = c.table[0, (c.lens[0] - c.cu[1] + j) // c.P], (c.lens[0] - c.cu[1] + j) % c.P
    held = c.vp[page, at, 1, 5].clone()
    c.vp[page, at, 1, 5] = value
    out, z2 = c.run()
    c.vp[page, at, 1, 5] = held
    want = clean.clone()
    sees = [t for t in range(c.cu[1]) if c.masks[t, j // 64] >> (j % 64) & 1]
    assert sees
    G = c.Hq // 2
    for t in sees:
        want[t, G:2 * G, 5] = value
    assert torch.equal(z, z2) and torch.equal(torch.nan_to_num(out, 3e4, 2e4, 1e4), torch.nan_to_num(want, 3e4, 2e4, 1e4))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,new", [(2, 40), (8, 40), (8, 70)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_rows_of_which_some_waves_meet_no_key(dtype, d, Hq, new, value):
    """Tokens that see themselves alone, in a request of no earlier ones."""
    for room in (0, 20000):
        c = with_room(TreeCase([0], [new], 0, Hq, 2, d, 16, dtype, seed=d), room)
        c.masks[:] = 0
        for t in range(new):
            c.masks[t, t // 64] = 1 << (t % 64) if t % 64 < 63 else -(1 << 63)
        for j in (2, 35, new - 1):
            check(c, j, value)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,new", [(2, 6), (8, 20), (8, 70)])
@pytest.mark.parametrize("place", ["prefix 0", "prefix 40", "own 5", "own 70", "own 590"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_beside_a_key_that_has_all_of_the_weight(dtype, d, Hq, new, place, value):
    """One earlier key's score is 250 above the others': their weights are 0 in 32 bits."""
    part, key = place.split()
    for room in (0, 20000):
        c = with_room(TreeCase([600], [new], 90, Hq, 2, d, 16, dtype, seed=d), room)
        c.q[..., 0] = 8.0
        high = 250.0 * math.sqrt(d) / 8.0
        if part == "prefix":
            c.pk[int(key), :, 0] = high
        else:
            c.kp[c.table[0, int(key) // 16], int(key) % 16, :, 0] = high
        for j in (0, new - 2):
            check(c, j, value)
