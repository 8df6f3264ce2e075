"""stem_tree_attn against exact attention in 64 bits, row by row, within bounds derived from its roundings (decode_util)."""
import math
import random

import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import tree_binding as tb

import tree_util as tu
from test_gpu_prefix_attn import BF, DEV, HF, SHAPES, Case

pytestmark = pytest.mark.gpu


class TreeCase(Case):
    def __init__(self, past, new, L, *args, branch=3, seed=0, **kw):
        super().__init__(past, new, L, *args, seed=seed, **kw)
        rng = random.Random(seed)
        rows = []
        for n in new:
            rows += [tu.words(s, tb.mask_words(self.max_new)) for s in tu.ancestors(tu.random_parents(rng, n, branch), n)[0]]
        rows += [[-1] * tb.mask_words(self.max_new)] * (self.q.shape[0] - len(rows))
        self.masks = torch.tensor(rows, dtype=torch.int64).view(self.q.shape[0], -1)

    def run(self, lse=True, out=None, cu=None, max_suffix=None, garbage=255):
        q, pk, pv = self.q.to(DEV), self.pk.to(DEV), self.pv.to(DEV)
        kp, vp = self.on_gpu(self.kp), self.on_gpu(self.vp)
        table, lens, cu = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (self.table.tolist(), self.lens, cu or self.cu))
        prefix = pk if self.L else None
        shape = db.PrefixShape.from_tensors(q, prefix, db.PageShape.from_tensors(kp, vp), table, self.max_new, self.max_suffix)
        space = torch.full((tb.stem_tree_attn_workspace_bytes(shape),), garbage, dtype=torch.uint8, device=DEV)   # NaN
        out = torch.full_like(q, 9.0) if out is None else out
        z = torch.full((self.Hq, q.shape[0]), 9.0, device=DEV) if lse else None
        tb.stem_tree_attn(shape, q, prefix, pv if self.L else None, kp, vp, table, lens, cu, self.masks.to(DEV), self.scale, out, z, space)
        return out.cpu(), z.cpu() if lse else None

    def check(self, out, z, cu=None, rows=None):
        want = tu.attention(self.q, self.pk if self.L else None, self.pv, self.kp, self.vp, self.table, self.lens, cu or self.cu, self.masks,
                            self.scale, self.max_new, self.max_suffix)
        for t in range(self.q.shape[0]) if rows is None else rows:
            if t not in want:
                assert (out[t] == 9.0).all() and (z is None or (z[:, t] == 9.0).all()), "row %d is nobody's" % t
                continue
            o, bound, lse, lse_bound = want[t]
            off = (out[t].double() - o).abs()
            assert (off <= bound).all(), "row %d: %g over" % (t, (off - bound).max())
            if z is not None:
                same = torch.isinf(lse) & (z[:, t].double() == lse)
                assert (same | ((z[:, t].double() - lse).abs() <= lse_bound)).all(), "row %d: lse" % t


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("past,new,L,P,padding", [
    ([0], [1], 1, 16, 0),                              # one key of the prefix, one of its own
    ([5, 0, 100], [4, 1, 3], 0, 16, 0),                # no prefix
    ([31, 32, 33, 127, 128, 129], [5, 1, 4, 2, 8, 3], 33, 32, 0),      # around whole tiles
    ([700, 3, 0, 64], [7, 20, 33, 1], 1000, 64, 0),
    ([40, 0, 17, 300], [3, 9, 0, 66], 257, 16, 4),     # two words, a request that waits, a padded batch
    ([15, 260], [140, 2], 300, 128, 1)])
def test_matches_exact_attention(dtype, Hq, Hkv, d, past, new, L, P, padding):
    c = TreeCase(past, new, L, Hq, Hkv, d, P, dtype, padding, seed=L + Hq + d, heads_first=P == 64)
    c.check(*c.run())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,new", [(4, 4, 1), (4, 4, 16), (8, 2, 4), (8, 2, 5), (8, 2, 16), (8, 2, 17), (8, 2, 33), (8, 1, 9), (7, 1, 40)])
@pytest.mark.parametrize("L", [0, 70])
def test_every_number_of_rows(d, Hq, Hkv, new, L):
    """Around each number of rows at which tiles change, over own keys in several parts."""
    c = TreeCase([1100, 0, 515], [new, new, max(new - 1, 0)], L, Hq, Hkv, d, 16, seed=new + d)
    c.check(*c.run())


def test_long_own_keys_and_wide_trees():
    c = TreeCase([5000, 20, 9000], [40, 3, 1], 0, 8, 2, 128, 16, seed=5, branch=5)
    c.check(*c.run())
    c = TreeCase([50], [1000], 0, 2, 1, 64, 16, seed=6, branch=300)
    c.check(*c.run(), rows=list(range(0, 1000, 37)) + [999])
    c = TreeCase([300] * 70, [2] * 70, 900, 4, 4, 64, 16, HF, seed=7)
    c.check(*c.run())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("past", [0, 7, 33])
def test_any_bits(d, past):
    """Masks that are no tree's: rows that see later tokens, not themselves, or none."""
    g = torch.Generator().manual_seed(d + past)
    for L in (0, 40):
        c = TreeCase([past, past + 100], [70, 9], L, 8, 2, d, 16, seed=past)
        c.masks = torch.randint(-(1 << 63), (1 << 63) - 1, c.masks.shape, generator=g, dtype=torch.int64)
        c.masks[3], c.masks[4], c.masks[75] = 0, -1, 0
        out, z = c.run()
        c.check(out, z)
        if past == 0 and L == 0:
            assert (out[3] == 0).all() and (z[:, 3] == -math.inf).all()


def test_one_token_that_does_not_see_itself():
    c = TreeCase([0, 3], [1, 1], 0, d=64)
    c.masks[:] = 0
    out, z = c.run()
    c.check(out, z)
    assert (out[0] == 0).all() and (z[:, 0] == -math.inf).all() and (z[:, 1] > -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("Hq,new,past,L", [(8, 6, 100, 50), (2, 3, 20, 0), (8, 20, 700, 0), (8, 90, 40, 300), (2, 12, 0, 0)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_is_not_finite_reaches_the_rows_that_see_it(dtype, Hq, new, past, L, value, d):
    """A new token's key or value, in a row that others see and in one that is its own alone."""
    c = TreeCase([past, 30], [new, 4], L, Hq, 2, d, 16, dtype, seed=new)
    then = c.run()
    c.check(*then)
    for j in (1, new - 1):
        sees = [bool(c.masks[t][j // 64] >> (j % 64) & 1) for t in range(new)] + [False] * 4
        page, at = c.table[0, (past + j) // 16], (past + j) % 16
        for x, columns in ((c.vp, [3]), (c.kp, range(d))):
            held = x[page, at].clone()
            x[page, at, 1, 3] = value
            out, z = c.run()
            x[page, at] = held
            heads = slice(Hq // 2, Hq)                 # those that read KV head 1
            for t in range(new + 4):
                if not sees[t]:
                    assert torch.equal(out[t], then[0][t]) and torch.equal(z[:, t], then[1][:, t]), (j, t)
                else:
                    assert torch.equal(out[t, :Hq // 2], then[0][t, :Hq // 2])
                    if x is c.vp:
                        assert not torch.isfinite(out[t, heads, 3]).any(), (j, t)
                        keep = [e for e in range(d) if e != 3]
                        assert torch.equal(out[t, heads][:, keep], then[0][t, heads][:, keep]) and torch.equal(z[:, t], then[1][:, t])
                        if value != value:
                            assert torch.isnan(out[t, heads, 3]).all()


@pytest.mark.parametrize("bad", [-1, 1 << 30])
@pytest.mark.parametrize("new", [3, 40])
def test_pages_that_are_none(bad, new):
    """Rows in pages that are not the cache's contribute nothing, in the middle of the earlier tokens and among the new ones."""
    c = TreeCase([200], [new], 33, 8, 2, 128, 16, seed=3)
    for entry in (4, 12, (200 + new - 1) // 16):
        c.table[0, entry] = bad
        c.check(*c.run())


def test_lens_outside_and_tokens_beyond():
    """Lengths outside 0 .. max_suffix count as the nearer; rows from max_new on stay; cu_new beyond the rows ends with them."""
    c = TreeCase([20, 40, 5], [6, 3, 4], 10, 4, 2, 64, 16)
    c.max_new = 4
    c.masks = c.masks[:, :1].contiguous()
    cu = [0, 6, 9, 50]
    c.check(*c.run(cu=cu), cu=cu)
    c = TreeCase([0, 4], [2, 3], 0, 4, 2, 64, 16)
    c.lens = [-7, 7]
    out, z = c.run()
    c.check(out, z)
    assert (out[:2] == 0).all()
    c.lens = [1, 7]                                    # two new tokens, of which only the later one is there
    c.check(*c.run())


def test_the_batch_and_the_workspace_do_not_matter():
    """The same bits whatever the workspace holds; no cross-talk between requests."""
    c = TreeCase([300, 10, 90], [9, 5, 30], 64, seed=4)
    a, b = c.run(garbage=255), c.run(garbage=0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.vp[c.table[1, 0]] = float("nan")
    d = c.run()
    keep = [t for t in range(44) if not 9 <= t < 14]
    assert torch.equal(a[0][keep], d[0][keep]) and torch.equal(a[1][:, keep], d[1][:, keep])


def test_chains_are_causal():
    """Masks of chains give what stem_prefix_attn gives, within both bounds."""
    c = TreeCase([200, 31], [9, 40], 100, branch=1, seed=8)
    tree, causal = c.run(), Case.run(c)
    c.check(*tree)
    Case.check(c, *causal)


def test_captured():
    c = TreeCase([100, 400, 33], [9, 20, 1], 77, seed=9)
    q, pk, pv, kp, vp = (x.to(DEV) for x in (c.q, c.pk, c.pv, c.kp, c.vp))
    table, lens, cu = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (c.table.tolist(), c.lens, c.cu))
    masks = c.masks.to(DEV)
    shape = db.PrefixShape.from_tensors(q, pk, db.PageShape.from_tensors(kp, vp), table, c.max_new, c.max_suffix)
    space = torch.empty(tb.stem_tree_attn_workspace_bytes(shape), dtype=torch.uint8, device=DEV)

    def run(out):
        tb.stem_tree_attn(shape, q, pk, pv, kp, vp, table, lens, cu, masks, c.scale, out, None, space)

    captured, eager = torch.zeros_like(q), torch.zeros_like(q)
    run(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(captured)
    for turn in range(4):
        q.copy_(torch.randn_like(q)), lens.sub_(1), masks.copy_(masks.flip(0))
        run(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, eager)
