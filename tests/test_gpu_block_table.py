"""stem_block_table against a plain account in Python: random steps, every kind of refusal, many requests, long steps, replays."""
import random

import pytest
import torch

from paper_2603_06274_amd import decode_binding as db

import decode_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Books:
    """The same cache kept twice: by the library on the GPU, by du.table_step here."""

    def __init__(self, R, P, W, N, cap, off=0, seed=0, in_place=True):
        r = random.Random(seed)
        self.R, self.P, self.W, self.N, self.cap, self.off = R, P, W, N, cap, off
        self.ring = list(range(N))
        r.shuffle(self.ring)
        self.state = [r.randrange(N), N]
        self.table = [[-7] * W for _ in range(R)]
        self.past = [0] * R
        t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        self.d_ring, self.d_state, self.d_table, self.d_past = t(self.ring), t(self.state), t(self.table), t(self.past)
        self.lens = self.d_past if in_place else torch.empty_like(self.d_past)
        self.state_out = self.d_state if in_place else torch.empty_like(self.d_state)
        self.cu, self.status = t([0] * (R + 1)), t([0] * 4)
        self.positions, self.slots = t([5] * max(cap, 1)), t([5] * max(cap, 1))
        self.shape = db.TableShape(R, P, N, W, cap, off)
        self.space = torch.empty(db.stem_block_table_workspace_bytes(self.shape), dtype=torch.uint8, device=DEV)
        self.in_place = in_place

    def call(self, new):
        db.stem_block_table(self.shape, self.d_past, new, self.d_state, self.d_ring, self.d_table, self.lens, self.state_out, self.cu,
                            self.positions, self.slots, self.status, self.space)

    def step(self, new, given=True):
        self.call(torch.tensor(new, dtype=torch.int32, device=DEV) if given else None)
        want = du.table_step(self.P, self.W, self.N, self.cap, self.off, self.past, new, self.ring, self.state, self.table)
        self.compare(want)
        if not self.in_place:
            self.d_past.copy_(self.lens), self.d_state.copy_(self.state_out)
        self.past, self.state = want["lens"], want["state"]
        return want

    def compare(self, want):
        for name, got in (("status", self.status), ("lens", self.lens), ("state", self.state_out), ("cu", self.cu),
                          ("positions", self.positions[:self.cap]), ("slots", self.slots[:self.cap])):
            assert got.tolist() == want[name], name
        assert self.d_ring.tolist() == self.ring and self.d_table.tolist() == self.table


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("R,P,W,N,cap,most_new", [
    (1, 16, 4, 4, 3, 3), (5, 16, 8, 30, 40, 20), (64, 64, 10, 500, 64, 1), (64, 16, 40, 2000, 5000, 200), (3, 256, 50, 120, 20000, 9000),
    (1024, 16, 6, 4000, 4096, 9), (1025, 16, 6, 4000, 4096, 9), (2500, 32, 4, 6000, 20000, 15)])
def test_steps_as_a_server_makes_them(R, P, W, N, cap, most_new, in_place):
    b = Books(R, P, W, N, cap, off=1000, seed=R, in_place=in_place)
    r = random.Random(N)
    refused = 0
    for step in range(12 if R < 1000 else 4):
        new = [r.choice([0, 1, 1, r.randint(0, most_new), -1 if r.random() < 0.3 else 1]) for _ in range(R)]
        if sum(max(n, 0) for n in new) > cap and step % 3:
            while sum(max(n, 0) for n in new) > cap:
                new[r.randrange(R)] = 0
        for x in range(R):                             # mostly within the table's rows
            if b.past[x] + max(new[x], 0) > W * P and r.random() < 0.9:
                new[x] = -1
        want = b.step(new)
        refused += any(want["status"])
        held = [p for x in range(R) for p in b.table[x][:-(-b.past[x] // P)]]
        free = [b.ring[(b.state[0] + i) % N] for i in range(b.state[1])]
        assert sorted(held + free) == list(range(N))   # every page once, whatever happened


def test_every_refusal_leaves_everything_as_it_was():
    b = Books(4, 16, 4, 8, 50, seed=1)
    b.step([30, 16, 1, 0])                             # 2 + 1 + 1 of 8 pages
    for new, what in (([0, 48, 32, 0], 0), ([35, 0, 0, 0], 1), ([0, 0, 63, 0], 2), ([0, 0, 64, 0], 1), ([34, 17, 0, 0], 2), ([2 ** 31 - 1] * 4, 1)):
        want = b.step(new)
        assert want["status"][what] > 0, (new, want["status"])
    b.d_past[2] = b.past[2] = -3                       # no length
    assert b.step([0, 1, 0, 0])["status"][1] == 1
    b.d_past[2] = b.past[2] = 1
    for state in ([8, 1], [-1, 1], [0, 9], [0, -1]):
        b.state = state
        b.d_state.copy_(torch.tensor(state))
        assert b.step([1, 0, 0, 0])["status"][3] == 1
    b.state = [3, 6]                                   # more free pages than there can be: those given back have no room
    b.d_state.copy_(torch.tensor(b.state))
    assert b.step([-1, -1, 0, 0])["status"][3] == 1


def test_one_token_each_without_new_lens_and_no_room_for_tokens():
    b = Books(70, 16, 3, 200, 70)
    for _ in range(20):
        b.step([1] * 70, given=False)
    c = Books(3, 16, 3, 9, 0)
    assert c.step([0, 0, 0])["status"] == [0, 0, 0, 0]
    assert c.step([1, 0, 0])["status"] == [0, 0, 1, 0]


def test_pages_that_are_none_give_no_slot():
    b = Books(2, 16, 3, 6, 40)
    b.step([16, 3])
    for bad in (-1, 6, 2 ** 31 - 1, -2 ** 31):
        b.table[0][0] = bad
        b.d_table[0, 0] = bad
        b.past = [10, 3]
        b.d_past.copy_(torch.tensor(b.past))
        want = b.step([4, 1])
        assert want["slots"][:4] == [-1] * 4 and want["slots"][4] >= 0


def test_sums_beyond_32_bits_refuse():
    """More new tokens in all than 32 bits hold, each of them within its row."""
    R, P, W = 40, 256, 1 << 19
    shape = db.TableShape(R, P, 10, W, 100, 0)
    t = lambda n, x: torch.full((n,), x, dtype=torch.int32, device=DEV)
    past, new, ring, state = t(R, 0), t(R, P * W), t(10, 0), torch.tensor([0, 10], dtype=torch.int32, device=DEV)
    table, lens, state_out, cu, pos, slots, status = t(R * W, -7), t(R, 9), t(2, 9), t(R + 1, 9), t(100, 9), t(100, 9), t(4, 9)
    space = torch.empty(db.stem_block_table_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    db.stem_block_table(shape, past, new, state, ring, table, lens, state_out, cu, pos, slots, status, space)
    assert status.tolist() == [R * W - 10, 0, 2 ** 31 - 1, 0]
    assert cu.tolist() == [0] * (R + 1) and slots.tolist() == [-1] * 100 and (table == -7).all() and lens.tolist() == [0] * R


@pytest.mark.parametrize("cap", [25, 700])             # one launch, two launches
def test_replays_go_on(cap):
    """A captured step, replayed with the books kept in place, beside eager steps of other books."""
    b, c = Books(20, 16, 6, 100, cap, seed=3), Books(20, 16, 6, 100, cap, seed=3)
    new = torch.ones(20, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.call(new)
    for step in range(30):
        fresh = [(-1 if (x + step) % 11 == 0 else (x + step) % 3) for x in range(20)]
        fresh = [f if sum(max(y, 0) for y in fresh[:x + 1]) <= 25 else 0 for x, f in enumerate(fresh)]
        new.copy_(torch.tensor(fresh, dtype=torch.int32))
        graph.replay()
        want = c.step(fresh)
        for x, y in ((b.slots, c.slots), (b.positions, c.positions), (b.d_table, c.d_table), (b.d_past, c.d_past),
                     (b.d_state, c.d_state), (b.d_ring, c.d_ring), (b.cu, c.cu), (b.status, c.status)):
            assert torch.equal(x, y), (step, want["status"])
