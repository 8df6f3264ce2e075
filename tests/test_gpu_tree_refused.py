"""An acceptance that is refused, and tried again when it can be done."""
import random

import pytest
import torch

from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode

import tree_util as tu

pytestmark = pytest.mark.gpu
DEV, BF = "cuda:0", torch.bfloat16


def test_tried_again():
    """Two caches that take the same steps, one of whose rings says nonsense for a moment: both end alike."""
    R, N, Hkv, d = 3, 9, 2, 64
    made = []
    for broken in (False, True):
        rng, g = random.Random(3), torch.Generator().manual_seed(3)
        prefix = torch.randn(40, Hkv, d, generator=g).to(BF).to(DEV)
        cache = PagedCache(R, 12, 16, 4, Hkv, d, tokens=R * N)
        dec = StemDecode(prefix, prefix.clone(), 4, cache, Rotary(d), max_new=N, tree=True)
        for step in range(3):
            new = [rng.randint(1, N) for _ in range(R)]
            parents = [p for n in new for p in tu.random_parents(rng, n, 2)]
            whole = [torch.tensor(x + [0] * (R * N - len(x)), dtype=torch.int32, device=DEV) for x in
                     (parents, [rng.randrange(2) for _ in parents], [rng.randrange(2) for _ in parents])]
            rows = [torch.randn(R * N, h, d, generator=g).to(BF).to(DEV) for h in (4, Hkv, Hkv)]
            dec.step(*rows, torch.tensor(new, dtype=torch.int32, device=DEV), parents=whole[0])
            if broken:
                then = [x.clone() for x in (cache.lens, cache.ring, cache.k_pages, cache.v_pages)]
                state = cache.ring_state.clone()
                cache.ring_state[0] = -1
                accepted, path, following = cache.accept(*whole)
                with pytest.raises(RuntimeError):
                    cache.accept(*whole)
                assert cache.accept_refused() == (0, 1) and accepted.tolist() == [0] * R and following.tolist() == [-1] * R
                for x, y in zip(then, (cache.lens, cache.ring, cache.k_pages, cache.v_pages)):
                    assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))       # (pages hold anything where nothing has been written)
                cache.ring_state.copy_(state)
            cache.accept(*whole)
            assert cache.accept_refused() == (0, 0)
            with pytest.raises(RuntimeError):
                cache.accept(*whole)
        made.append((cache.lens, cache.ring_state, cache.ring, cache.table, cache.accepted, cache.path, dec.out))
    for x, y in zip(*made):
        assert torch.equal(x, y)


def test_a_replayed_step_of_drafts_behind_an_eager_one_of_single_tokens():
    R, N, Hkv, d = 3, 7, 2, 64
    g = torch.Generator().manual_seed(5)
    prefix = torch.randn(40, Hkv, d, generator=g).to(BF).to(DEV)
    cache = PagedCache(R, 24, 16, 8, Hkv, d, tokens=R * N)
    drafts, single = (StemDecode(prefix, prefix.clone(), 4, cache, Rotary(d), max_new=n, tree=True) for n in (N, 1))
    rows = [torch.randn(R * N, h, d, generator=g).to(BF).to(DEV) for h in (4, Hkv, Hkv)]
    ones, chain = (torch.tensor(x * R, dtype=torch.int32, device=DEV) for x in ([1], [-1, *range(N - 1)]))
    new, ids = torch.zeros(R, dtype=torch.int32, device=DEV), torch.zeros(R * N, dtype=torch.int64, device=DEV)
    drafts.step(*rows, new, parents=chain)             # (of nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        drafts.step(*rows, new, parents=chain)
    new.fill_(N)
    for turn in range(3):
        single.step(*rows, ones)
        graph.replay()
        accepted = cache.accept(chain, ids, ids)[0]    # every draft is the model's choice
        assert cache.accept_refused() == (0, 0) and accepted.tolist() == [N] * R and cache.lens.tolist() == [(turn + 1) * (N + 1)] * R
