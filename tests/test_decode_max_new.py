"""Steps with more new tokens of a request than their attention takes: refused like those without room, in one launch and in two."""
import ctypes

import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import PagedCache, StemDecode

DEV = "cuda:0"


def test_a_bound_below_zero_is_refused():
    n = ctypes.c_size_t()
    for max_new, status in ((0, sb.STEM_OK), (7, sb.STEM_OK), (2 ** 31 - 1, sb.STEM_OK), (-1, sb.STEM_ERR_INVALID_ARG)):
        shape = db.TableShape(2, 16, 10, 4, 8, max_new=max_new)
        assert db.lib().stem_block_table_workspace_bytes(shape.ref, ctypes.byref(n)) == status


@pytest.mark.gpu
@pytest.mark.parametrize("R,tokens", [(3, 40), (3, 4000), (1100, 4000)])
def test_more_tokens_than_allowed(R, tokens):
    cache = PagedCache(R, 4000, 16, 40, 1, 64, tokens=tokens, device=DEV)
    new = torch.zeros(R, dtype=torch.int32, device=DEV)

    def step(lens, max_new):
        new.zero_()
        new[:3] = torch.tensor(lens, dtype=torch.int32)
        cache.advance(new, max_new)
        return cache.refused(), cache.lens[:3].tolist(), int(cache.cu_new[-1])

    assert step([5, 5, 2], 5) == ((0, 0, 0, 0), [5, 5, 2], 12)
    before = [x.clone() for x in (cache.table, cache.ring, cache.ring_state, cache.lens)]
    assert step([6, 1, 7], 5) == ((0, 2, 0, 0), [5, 5, 2], 0)
    assert (cache.slots == -1).all() and (cache.positions == 0).all()
    assert all(torch.equal(x, y) for x, y in zip(before, (cache.table, cache.ring, cache.ring_state, cache.lens)))
    assert step([6, -1, 7], 7) == ((0, 0, 0, 0), [11, 0, 9], 13)   # a finished request has none
    assert step([20, 0, 0], 0) == ((0, 0, 0, 0), [31, 0, 9], 20)   # any number


@pytest.mark.gpu
def test_a_step_takes_no_more_than_its_attention():
    g = torch.Generator().manual_seed(1)
    rows = lambda n, h: torch.randn(n, h, 64, generator=g).to(torch.bfloat16).to(DEV)
    pk = rows(30, 1)
    cache = PagedCache(2, 8, 16, 4, 1, 64, tokens=6, position_offset=30, device=DEV)
    dec = StemDecode(pk, pk, 2, cache, max_new=2)
    given = rows(6, 2), rows(6, 1), rows(6, 1)
    dec.out.fill_(9.0)
    dec.step(*given, torch.tensor([3, 1], dtype=torch.int32, device=DEV))
    assert cache.refused() == (0, 1, 0, 0) and cache.lens.tolist() == [0, 0] and (dec.out == 9.0).all()
    dec.step(*given, torch.tensor([2, 1], dtype=torch.int32, device=DEV))
    assert cache.refused() == (0, 0, 0, 0) and cache.lens.tolist() == [2, 1] and not (dec.out[:3] == 9.0).any()
    cache.advance(torch.tensor([3, 1], dtype=torch.int32, device=DEV))          # (by itself, any number)
    assert cache.refused() == (0, 0, 0, 0) and cache.lens.tolist() == [5, 2]
