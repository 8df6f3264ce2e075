"""Decoding behind a prompt that was pre-filled in chunks, its queries and keys turned before the calls."""
import pytest
import torch

from paper_2603_06274_amd.decode import PagedCache, Rotary
from paper_2603_06274_amd.prefill import StemPrefill

pytestmark = pytest.mark.gpu
BF, DEV = torch.bfloat16, "cuda:0"


def test_chunks_then_steps():
    g = torch.Generator().manual_seed(1)
    rows = lambda n, h: torch.randn(n, h, 64, generator=g).to(BF).to(DEV)
    T, at = 320, 192
    q, k, v = rows(T, 2), rows(T, 1), rows(T, 1)
    r = Rotary(64, theta=1000.0)
    kw = dict(n_sink=1, n_local=1)
    whole = StemPrefill(q, k, v, [0, T], 64, [9], 1.0, rotary=r, **kw)
    whole.run()
    tq, tk = r.apply(q, k, torch.arange(T, dtype=torch.int32, device=DEV))
    first = StemPrefill(tq[:at], tk, v, [0, T], 64, [9], 1.0, chunk=([0], [at]), **kw)
    last = StemPrefill(tq[at:], tk, v, [0, T], 64, [9], 1.0, chunk=([at], [T]), workspace=first.workspace, **kw)
    first.run(), last.run()
    make = lambda **kw: PagedCache(2, 4, 16, 2, 1, 64, **kw)
    caches = [make(), make(), make(position_offset=T)]
    decoders = [whole.decode(caches[0]), last.decode(caches[1], rotary=r), last.decode(caches[2], rotary=r)]
    for _ in range(2):
        step = rows(2, 2), rows(2, 1), rows(2, 1)
        outs = [d.step(*step) for d in decoders]
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        assert torch.equal(caches[0].k_pages[caches[0].table[0, 0]][:1], caches[1].k_pages[caches[1].table[0, 0]][:1])
    # rows that come turned already
    cache = make(position_offset=T)
    plain = last.decode(cache)
    step = rows(2, 2), rows(2, 1), rows(2, 1)
    turned = r.apply(*step[:2], torch.full((2,), T, dtype=torch.int32, device=DEV))
    assert torch.equal(plain.step(*turned, step[2]), last.decode(make(), rotary=r).step(*step))
    with pytest.raises(ValueError):                                # places other than behind the prompt
        last.decode(make(position_offset=T - 1), rotary=r)
    with pytest.raises(ValueError):                                # keys turned by other positions
        whole.decode(make(), rotary=Rotary(64))
