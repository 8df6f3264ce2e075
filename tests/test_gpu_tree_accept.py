"""stem_tree_accept and stem_tree_commit against their definitions: walks, lengths, pages given back, rows moved."""
import random

import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import tree_binding as tb

import tree_util as tu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def whole(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


class Books:
    """Random requests behind a step of drafts from few token numbers, so that siblings are often alike."""

    def __init__(self, rng, past, new, P, branch, padding=0, spare_pages=4, vocabulary=3):
        self.P, self.past, self.new = P, past, new
        self.lens = [p + n for p, n in zip(past, new)]
        self.cu = [sum(new[:r]) for r in range(len(new) + 1)]
        self.T = self.cu[-1] + padding
        self.parents = [p for n in new for p in tu.random_parents(rng, n, branch)] + [0] * padding
        self.drafts, self.targets = ([rng.randrange(vocabulary) for _ in range(self.T)] for _ in range(2))
        held = [-(-n // P) for n in self.lens]
        self.W, self.N = max(held + [0]) + 2, sum(held) + spare_pages + 3
        order = list(range(self.N))
        rng.shuffle(order)
        self.table, at = [], 0
        for h in held:
            self.table.append(order[at:at + h] + [-1] * (self.W - h))
            at += h
        self.state = [rng.randrange(self.N), spare_pages]
        self.ring = [-7] * self.N
        for i in range(spare_pages):
            self.ring[(self.state[0] + i) % self.N] = order[at + i]
        self.max_new = max(new + [1])

    def run(self, ids=torch.int64, in_place=False):
        shape = tb.AcceptShape(len(self.new), self.T, self.max_new, self.P, self.N, self.W)
        space = torch.full((tb.stem_tree_accept_workspace_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
        lens, state, ring, table = whole(self.lens), whole(self.state), whole(self.ring), whole(self.table)
        lens_out, state_out = (lens, state) if in_place else (torch.full_like(lens, 77), torch.full_like(state, 77))
        accepted, path, status = torch.full_like(lens, 77), torch.full((self.T,), 77, dtype=torch.int32, device=DEV), whole([77, 77])
        following = torch.full((len(self.new),), 77, dtype=ids, device=DEV)
        tb.stem_tree_accept(shape, whole(self.parents), whole(self.drafts, ids), whole(self.targets, ids), whole(self.cu), lens, state, ring,
                            table, lens_out, state_out, accepted, path, following, status, space)
        assert table.tolist() == self.table
        return dict(lens=lens_out, state=state_out, ring=ring, accepted=accepted, path=path, next=following, status=status)

    def check(self, got):
        ring = list(self.ring)
        want = tu.accept(self.P, self.W, self.N, self.max_new, self.parents, self.drafts, self.targets, self.cu, self.lens, ring, self.state,
                         self.table)
        for x in ("status", "lens", "state", "accepted", "next"):
            assert got[x].tolist() == want[x], x
        assert got["ring"].tolist() == ring
        path = got["path"].tolist()
        assert path == [want["path"].get(t, 77) for t in range(self.T)]
        return want


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("requests,most_new,most_past,P,branch", [
    (1, 1, 5, 16, 1), (1, 40, 0, 16, 3), (7, 9, 100, 16, 1), (64, 16, 300, 64, 4), (64, 64, 300, 16, 2), (65, 65, 30, 32, 9),
    (3, 1024, 50, 16, 1), (3, 1000, 50, 256, 500), (1500, 6, 40, 16, 2),
    (16, 30, 100, 16, 3), (17, 30, 100, 16, 3), (16, 256, 100, 16, 2), (16, 257, 100, 16, 2), (6, 900, 100, 32, 4)])
def test_matches_its_definition(ids, requests, most_new, most_past, P, branch):
    for seed in range(3):
        rng = random.Random(seed * 100 + requests)
        b = Books(rng, [rng.randint(0, most_past) for _ in range(requests)], [rng.randint(0, most_new) for _ in range(requests)], P, branch,
                  padding=seed, vocabulary=1 + seed)
        want = b.check(b.run(ids, in_place=seed == 1))
        assert want["status"] == [0, 0]


def test_large_token_numbers():
    """64-bit numbers that agree in their lower half are different ones."""
    b = Books(random.Random(1), [3], [4], 16, 1)
    b.drafts, b.targets = [0, 5 + (1 << 40), 6, 7], [5 + (1 << 40), 6 + (1 << 33), 7, 8]
    want = b.check(b.run())
    assert want["accepted"] == [2] and want["next"] == [6 + (1 << 33)]


def test_parents_that_are_none_and_several_roots():
    b = Books(random.Random(2), [3, 20], [5, 4], 16, 1)
    b.parents, b.drafts, b.targets = [-1, 7, -1, 3, 1 << 30, 0, 0, 0, 1], [1] * 9, [1] * 9
    want = b.check(b.run())
    assert want["accepted"] == [1, 3]


@pytest.mark.parametrize("what", ["new", "lens", "row", "state", "count", "room"])
def test_refused(what):
    """Nothing moves, and the status says why."""
    for requests in (5, 1200):
        rng = random.Random(3)
        b = Books(rng, [20] * requests, [20] * requests, 16, 2)
        if what == "new":
            b.max_new = 19
        elif what == "lens":
            b.lens[1] = 19
        elif what == "row":
            b.lens[2] = b.W * b.P + 1
        elif what == "state":
            b.state[0] = b.N
        elif what == "count":
            b.state[1] = -1
        else:
            b.state[1] = b.N
        want = b.check(b.run(in_place=True))
        assert any(want["status"]) and set(want["accepted"]) == {0}


def test_no_tokens():
    b = Books(random.Random(4), [0, 5], [0, 0], 16, 1)
    want = b.check(b.run())
    assert want["status"] == [0, 0] and want["lens"] == [0, 5]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("Hkv,d,P,new", [(8, 128, 16, [9, 0, 30]), (1, 8, 16, [5]), (3, 72, 64, [17, 64, 100]), (2, 1024, 32, [1, 40])])
def test_commit(dtype, Hkv, d, P, new):
    """Rows move up along random paths, also by less than a turn of the kernel; everything else stays."""
    rng = random.Random(d)
    g = torch.Generator().manual_seed(d)
    T, cu = sum(new) + 2, [sum(new[:r]) for r in range(len(new) + 1)]
    N = -(-T // P) + 2
    kp, vp = (torch.randn(N, P, Hkv, d + 8, generator=g).to(dtype).to(DEV)[..., :d] for _ in range(2))
    slots = torch.randperm(N * P, generator=g)[:T].tolist()
    for t in (3, T - 1):
        slots[t] = -1 if t == 3 else N * P
    path = [77] * T
    for r, n in enumerate(new):
        kept = sorted(rng.sample(range(n), rng.randint(0, n))) if n else []
        for k in range(n):
            path[cu[r] + k] = kept[k] if k < len(kept) else -1
    want = []
    for x in (kp, vp):
        flat, then = x.reshape(N * P, Hkv, d).clone(), x.reshape(N * P, Hkv, d)
        for r, n in enumerate(new):
            for k in range(n):
                i = path[cu[r] + k]
                if i < 0:
                    break
                to, of = slots[cu[r] + k], slots[cu[r] + i]
                if 0 <= to < N * P and 0 <= of < N * P:
                    flat[to] = then[of]
        want.append(flat)
    shape = tb.AcceptShape(len(new), T, max(new), P, N, 4)
    tb.stem_tree_commit(shape, db.PageShape.from_tensors(kp, vp), whole(path), whole(slots), whole(cu), kp, vp)
    for x, y in zip((kp, vp), want):
        assert torch.equal(x.reshape(N * P, Hkv, d), y)


def test_commit_stops_at_what_is_no_number():
    kp = torch.arange(64 * 8, device=DEV, dtype=torch.float32).view(4, 16, 1, 8).contiguous()
    vp, then = kp.clone(), kp.clone()
    shape = tb.AcceptShape(2, 8, 4, 16, 4, 4)
    slots = whole([0, 1, 2, 3, 20, 21, 22, 23])
    tb.stem_tree_commit(shape, db.PageShape.from_tensors(kp, vp), whole([1, 4, 3, 3, 2, 1 << 30, 0, 0]), slots, whole([0, 4, 8]), kp, vp)
    flat = then.view(64, 8).clone()
    flat[0], flat[20] = then.view(64, 8)[1], then.view(64, 8)[22]
    assert torch.equal(kp.view(64, 8), flat) and torch.equal(vp.view(64, 8), flat)
