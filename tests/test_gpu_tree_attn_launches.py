"""The attention of drafted tokens in one launch and in two: by what the table's rows have room for, with the same tokens.  Row tiles of all
sizes, prefix and own keys, several parts joined by rows of many requests, values that are not finite."""
import math

import pytest
import torch

from test_gpu_prefix_attn import BF, DEV, HF
from test_gpu_tree_attn import TreeCase

pytestmark = pytest.mark.gpu


def with_room(c, keys):
    """The case with table rows of `keys` tokens and more."""
    entries = -(-keys // c.P)
    c.table = torch.cat([c.table, torch.full((c.table.shape[0], max(entries - c.table.shape[1], 0)), -1, dtype=c.table.dtype)], dim=1)
    c.max_suffix = c.table.shape[1] * c.P
    return c


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,new", [(4, 4, [1, 3]), (8, 2, [4, 0, 2]), (8, 2, [16, 5, 9]), (8, 2, [33, 1]), (7, 1, [40, 12]), (4, 1, [70])])
@pytest.mark.parametrize("L", [0, 90, 700])
def test_both(dtype, d, Hq, Hkv, new, L):
    past = [31, 200, 0][:len(new)]
    for room in (0, 20000):
        c = with_room(TreeCase(past, new, L, Hq, Hkv, d, 16, dtype, 2, seed=L + d), room)
        c.check(*c.run())


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 32, 8), (256, 4, 4)])
def test_many_requests_of_few_tokens(d, Hq, Hkv):
    """Rows by the call's tokens rather than by what each request might have: the largest has far more than the others."""
    new = [40] + [1, 2, 0] * 12
    past = [(r * 37) % 150 for r in range(len(new))]
    for room in (0, 20000):
        c = with_room(TreeCase(past, new, 130, Hq, Hkv, d, 16, BF, 3, seed=d), room)
        c.check(*c.run(), rows=list(range(0, c.q.shape[0], 5)) + list(range(c.q.shape[0] - 3, c.q.shape[0])))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d,new", [(64, 20), (128, 20), (256, 9)])
@pytest.mark.parametrize("L", [0, 90])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, d, new, L, value):
    for room in (0, 20000):
        c = with_room(TreeCase([40, 10], [new, new], L, 8, 2, d, 16, dtype, seed=d), room)
        clean, z = c.run()
        page, at = c.table[0, (40 + new - 3) // 16], (40 + new - 3) % 16       # new token number new - 3
        c.vp[page, at, 1, 5] = value
        out, z2 = c.run()
        sees = [t for t in range(new) if c.masks[t, 0] >> (new - 3) & 1]
        assert sees == [t for t in sees if t >= new - 3] and sees
        others = [t for t in range(2 * new) if t not in sees]
        assert torch.equal(out[others], clean[others]) and torch.equal(z, z2)
        G = 4
        hit = torch.zeros(8, d, dtype=torch.bool)
        hit[G:2 * G, 5] = True
        for t in sees:
            assert not out[t][hit].isfinite().any() and torch.equal(out[t][~hit], clean[t][~hit])


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_that_see_nothing(d):
    for room in (0, 20000):
        c = with_room(TreeCase([0, 0], [20, 3], 0, 8, 2, d, 16, BF, seed=d), room)
        c.masks[::2] = 0
        out, z = c.run()
        c.check(out, z)
        assert (out[:23:2] == 0).all() and (z[:, :23:2] == -math.inf).all()
