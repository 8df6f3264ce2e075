"""Where the positions of new tokens begin: behind the prefix, unless the cache was made with another place."""
import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode
from paper_2603_06274_amd.prefill import StemPrefill

BF, DEV = torch.bfloat16, "cuda:0"


def rows(g, n, h, dev):
    return torch.randn(n, h, 64, generator=g).to(BF).to(dev)


def offset(cache):
    return cache.shape.c.position_offset


def test_a_cache_begins_behind_the_first_prefix(monkeypatch):
    monkeypatch.setattr(db, "stem_prefix_attn_workspace_bytes", lambda shape: 256)
    monkeypatch.setattr(db, "stem_block_table", lambda *a: None)
    make = lambda **kw: PagedCache(2, 4, 16, 2, 1, 64, device="cpu", **kw)
    g = torch.Generator().manual_seed(1)
    long, short = rows(g, 300, 1, "cpu"), rows(g, 50, 1, "cpu")
    r = Rotary(64, device="cpu")
    cache = make()
    assert offset(cache) == 0
    StemDecode(long, long, 2, cache)                               # no positions: whatever the cache has
    assert offset(cache) == 0
    StemDecode(long, long, 2, cache, r)
    assert offset(cache) == 300
    StemDecode(long, long, 2, cache, r)                            # another layer of the same prefix
    with pytest.raises(ValueError):
        StemDecode(short, short, 2, cache, r)
    assert offset(cache) == 300
    begun = make()
    begun.advance()
    with pytest.raises(ValueError):                                # its first tokens stand at 0 and on
        StemDecode(short, short, 2, begun, r)
    for given in (0, 50, 77):                                      # as it was asked for
        cache = make(position_offset=given)
        StemDecode(short, short, 2, cache, r)
        assert offset(cache) == given
    far = PagedCache(2, 4, 256, (2 ** 31 - 1) // 256, 1, 64, device="cpu")
    with pytest.raises(sb.StemError):                              # positions beyond 32 bits
        StemDecode(long, long, 2, far, r)
    assert offset(far) == 0


@pytest.mark.gpu
def test_new_tokens_stand_behind_the_prefix():
    g = torch.Generator().manual_seed(2)
    q, k, v = rows(g, 300, 2, DEV), rows(g, 300, 1, DEV), rows(g, 300, 1, DEV)
    r = Rotary(64, theta=500.0)
    pf = StemPrefill(q, k, v, [0, 300], 64, [9], 1.0, n_sink=1, n_local=1, rotary=r)
    pf.run()
    make = lambda **kw: PagedCache(2, 4, 16, 2, 1, 64, **kw)
    told, untold, direct = make(position_offset=300), make(), make()
    decoders = [pf.decode(told), pf.decode(untold), StemDecode(pf.k, v, 2, direct, r)]
    for _ in range(3):
        step = rows(g, 2, 2, DEV), rows(g, 2, 1, DEV), rows(g, 2, 1, DEV)
        outs = [d.step(*step) for d in decoders]
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert untold.positions.tolist() == [302, 302] == direct.positions.tolist()
    with pytest.raises(ValueError):
        pf.decode(make(position_offset=0))
