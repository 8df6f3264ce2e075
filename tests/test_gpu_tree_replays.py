"""Steps in a replayed graph with acceptances outside of it, and the other way round: each is that of the step before it."""
import random

import pytest
import torch

from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode

import tree_util as tu

pytestmark = pytest.mark.gpu
DEV, BF = "cuda:0", torch.bfloat16
HQ, HKV, D, R, N = 4, 2, 64, 3, 7


def whole(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Steps:
    def __init__(self, prefix):
        self.dec = StemDecode(prefix, prefix.clone(), HQ, PagedCache(R, 40, 16, 12, HKV, D, tokens=R * N), Rotary(D), max_new=N, tree=True)
        T = self.dec.cache.tokens
        self.x = [torch.zeros(T, h, D, dtype=BF, device=DEV) for h in (HQ, HKV, HKV)]
        self.new, self.parents, self.ids, self.choice = whole([0] * R), whole([-1] * T), whole([0] * T), whole([0] * T)

    def load(self, rng, g):
        lens = [rng.randint(0, N) for _ in range(R)]
        parents = [p for n in lens for p in tu.random_parents(rng, n, 2)]
        T = self.dec.cache.tokens
        for dst, src in ((self.new, lens), (self.parents, parents + [-1] * (T - len(parents))),
                         (self.ids, [rng.randrange(2) for _ in range(T)]), (self.choice, [rng.randrange(2) for _ in range(T)])):
            dst.copy_(whole(src))
        for t in self.x:
            t.copy_(torch.randn(t.shape, generator=g).to(BF))

    def step(self):
        self.dec.step(*self.x, self.new, parents=self.parents)

    def accept(self):
        self.dec.cache.accept(self.parents, self.ids, self.choice)


@pytest.mark.parametrize("captured", ["step", "accept"])
def test_one_in_a_graph_and_the_other_not(captured):
    prefix = torch.randn(90, HKV, D, generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    made = [Steps(prefix) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    for m in made:                                     # (a step of nothing)
        m.step()
        m.accept()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        made[0].step() if captured == "step" else made[0].accept()
    streams = [(random.Random(5), torch.Generator().manual_seed(5)) for _ in made]
    for _ in range(6):
        for m, s in zip(made, streams):
            m.load(*s)
            if m is made[0] and captured == "step":
                graph.replay()
            else:
                m.step()
            torch.cuda.synchronize()
            if m is made[0] and captured == "accept":
                graph.replay()
            else:
                m.accept()
        a, b = (m.dec.cache for m in made)
        for s, t in ((a.lens, b.lens), (a.ring, b.ring), (a.ring_state, b.ring_state), (a.table, b.table), (a.path, b.path),
                     (a.accepted, b.accepted), (made[0].dec.out, made[1].dec.out)):
            assert torch.equal(s, t)
    with pytest.raises(RuntimeError):                  # where nothing has been captured a second time is seen
        made[1].accept()
