"""Steps that cannot be done are refused before anything of them is enqueued: lengths, table and free pages stay as they were, and so does
what the cache holds.  On the host the library's calls are recorded; on the GPU the books are looked at."""
import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode

BF = torch.bfloat16
REFUSED = (ValueError, sb.StemError)


class Books:
    def __init__(self, dev, calls):
        self.dev, self.calls = dev, calls
        g = torch.Generator().manual_seed(3)
        self.rows = lambda n, h, d=64: torch.randn(n, h, d, generator=g).to(BF).to(dev)

    def cache(self, **kw):
        return PagedCache(2, 4, 16, 2, 1, 64, device=self.dev, **kw)

    def untouched(self, cache, lens=(0, 0)):
        assert not self.calls
        assert cache.lens.tolist() == list(lens) and cache.ring_state.tolist() == [0, 4] and (cache.table == -1).all()


@pytest.fixture(params=["cpu", pytest.param("cuda:0", marks=pytest.mark.gpu)])
def books(request, monkeypatch):
    calls = []
    if request.param == "cpu":
        monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
        monkeypatch.setattr(sb, "_raw_stream", lambda dev: 0)
        monkeypatch.setattr(db, "stem_prefix_attn_workspace_bytes", lambda shape: 256)
        for name in ("stem_block_table", "stem_rotary_append", "stem_prefix_attn"):
            monkeypatch.setattr(db, name, lambda *a, _n=name: calls.append(_n))
    return Books(request.param, calls)


def test_rows_that_the_library_would_refuse(books):
    rows = books.rows
    cache = books.cache(position_offset=50)
    pk = rows(50, 1)
    dec = StemDecode(pk, pk, 4, cache, Rotary(64, device=books.dev))
    q, k, v = rows(2, 4), rows(2, 1), rows(2, 1)

    def slice_of(t, token, at):
        """The same values in a buffer of `token` elements per row, from element `at` on."""
        room = torch.zeros(2 * token + at, dtype=BF, device=books.dev)
        out = room[at:].as_strided(t.shape, (token, 64, 1), at)
        out.copy_(t)
        return out

    bad = [(q, slice_of(k, 196, 0), slice_of(v, 196, 0)),          # strides that are not whole 16 bytes
           (q, slice_of(k, 192, 4), slice_of(v, 192, 0)), (q, slice_of(k, 192, 0), slice_of(v, 192, 4)),   # nor addresses
           (slice_of(q, 260, 0), k, v), (slice_of(q, 256, 4), k, v),
           (q, k[:1].expand(2, 1, 64), v[:1].expand(2, 1, 64)),    # one row for every request
           (q[:, :1].expand(2, 4, 64), k, v), (q[:1].expand(2, 4, 64), k, v)]
    for given in bad:
        with pytest.raises(REFUSED):
            dec.step(*given)
        books.untouched(cache)
    if books.dev == "cpu":
        return
    first = dec.step(q, k, v).clone()                              # and then it goes on as if nothing had been
    assert cache.lens.tolist() == [1, 1]
    again = StemDecode(pk, pk, 4, books.cache(position_offset=50), Rotary(64, device=books.dev))
    assert torch.equal(first, again.step(q, slice_of(k, 192, 8), slice_of(v, 192, 8)))


def test_a_prefix_that_cannot_be_attended_to(books):
    rows, wide = books.rows, books.rows(50, 3)
    for pk, pv in ((rows(50, 1), wide[:, 1:2]), (wide[:, :1], rows(50, 1)), (rows(50, 1), rows(49, 1)), (rows(50, 1), rows(50, 1).half()),
                   (rows(50, 1), rows(50, 1, 128)[:, :, :64]), (rows(51, 1).flatten()[4:3204].view(50, 1, 64), rows(50, 1)),
                   (rows(50, 1), rows(51, 1).flatten()[4:3204].view(50, 1, 64))):
        cache = books.cache()
        with pytest.raises(REFUSED):
            StemDecode(pk, pv, 4, cache)
        books.untouched(cache)
    StemDecode(wide[:, :1], wide[:, 1:2], 4, books.cache())        # views of one projection are fine


def test_scales_that_are_none(books):
    pk = books.rows(50, 1)
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e39, 1e-60):
        with pytest.raises(REFUSED):
            StemDecode(pk, pk, 4, books.cache(), softmax_scale=scale)


def test_positions_that_do_not_go_with_the_cache(books):
    for bad in (dict(rotary_dim=128), dict(rotary_dim=66), dict(layout="third")):
        with pytest.raises(REFUSED):
            Rotary(64, device=books.dev, **bad)
    for head_dim in (68, 2048):
        with pytest.raises(REFUSED):
            Rotary(head_dim, 64, device=books.dev)
    pk, cache = books.rows(50, 1), books.cache(position_offset=50)
    elsewhere = Rotary(64, device="meta" if books.dev == "cpu" else "cpu")
    with pytest.raises(REFUSED):
        StemDecode(pk, pk, 4, cache, elsewhere)
    with pytest.raises(REFUSED):
        cache.append(elsewhere, None, books.rows(2, 1), books.rows(2, 1))
    books.untouched(cache)


def test_sizes_beyond_the_library(books):
    pk = books.rows(50, 1)
    with pytest.raises(REFUSED):
        PagedCache(2, 4, 16, 2, 1, 64, tokens=1 << 24, device=books.dev)
    with pytest.raises(REFUSED):                                   # query heads and those of keys and values together
        StemDecode(pk, pk, 65534, books.cache())


def test_lengths_that_are_none(books):
    pk, cache = books.rows(50, 1), books.cache()
    if books.dev == "cpu":
        return                                                     # (the recorders look at nothing)
    dec = StemDecode(pk, pk, 4, cache)
    given = books.rows(2, 4), books.rows(2, 1), books.rows(2, 1)
    for new in (torch.ones(2, dtype=torch.int64, device=books.dev), torch.ones(1, dtype=torch.int32, device=books.dev),
                torch.ones(2, dtype=torch.int32), torch.ones(4, dtype=torch.int32, device=books.dev)[::2]):
        with pytest.raises(REFUSED):
            dec.step(*given, new)
        books.untouched(cache)
