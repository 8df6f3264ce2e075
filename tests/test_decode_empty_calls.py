"""Calls without tokens, with tensors that have none (whose address is 0): they do nothing and are not refused."""
import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import PagedCache, Rotary, StemDecode

BF = torch.bfloat16


@pytest.fixture(params=["cpu", pytest.param("cuda:0", marks=pytest.mark.gpu)])
def dev(request, monkeypatch):
    if request.param == "cpu":                         # (nothing is launched, so tensors of the host will do)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
        monkeypatch.setattr(sb, "_raw_stream", lambda dev: 0)
    return request.param


def none(*sizes, dtype=BF, dev="cpu"):
    return torch.empty(0, *sizes, dtype=dtype, device=dev)


def test_rotary(dev):
    r = Rotary(64, device=dev)
    q, k, pos = none(4, 64, dev=dev), none(2, 64, dev=dev), none(dtype=torch.int32, dev=dev)
    for given in ((q, k), (q, None), (None, k)):
        for f in (r.apply, r.backward):
            for x, y in zip(f(*given, pos), given):
                assert (x is None and y is None) or x.shape == y.shape


@pytest.mark.parametrize("pages", [0, 3])
def test_append(dev, pages):
    q, k, pos = none(4, 64, dev=dev), none(2, 64, dev=dev), none(dtype=torch.int32, dev=dev)
    kp, vp = (torch.full((pages, 16, 2, 64), 3.0, dtype=BF, device=dev) for _ in range(2))
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    for rows in (q, None):
        db.stem_rotary_append(db.RotaryShape.from_tensors(rows, k, 64), db.PageShape.from_tensors(kp, vp), rows, k, k.clone(), pos, pos,
                              turns.to(dev), factor, rows, kp, vp)
    assert (kp == 3.0).all() and (vp == 3.0).all()


@pytest.mark.gpu
def test_a_cache_without_pages():
    q, pos = torch.zeros(3, 2, 64, dtype=BF, device="cuda:0"), torch.zeros(3, dtype=torch.int32, device="cuda:0")
    kp = torch.empty(0, 16, 2, 64, dtype=BF, device="cuda:0")
    turns, factor = db.stem_rotary_frequencies(64, 10000.0)
    db.stem_rotary_append(db.RotaryShape.from_tensors(None, q, 64), db.PageShape.from_tensors(kp, kp.clone()), None, q, q.clone(), pos,
                          pos, turns.to("cuda:0"), factor, None, kp, kp.clone())


@pytest.mark.gpu
def test_attention_and_steps():
    dev = "cuda:0"
    pk = torch.randn(100, 2, 64, device=dev).to(BF)
    cache = PagedCache(3, 4, 16, 2, 2, 64, tokens=0, position_offset=100, device=dev)
    dec = StemDecode(pk, pk.clone(), 4, cache, Rotary(64, device=dev), want_lse=True)
    new = torch.tensor([0, 0, -1], dtype=torch.int32, device=dev)
    assert dec.step(none(4, 64, dev=dev), none(2, 64, dev=dev), none(2, 64, dev=dev), new).shape == (0, 4, 64)
    assert cache.refused() == (0, 0, 0, 0)


def test_attention_of_no_rows():
    """Through the C ABI: a prefix and no row."""
    import ctypes
    c = db.stem_prefix_shape(db.STEM_BF16, 4, 2, 64, 3, 0, 1, 100, 0, 0, 256, 64, 128, 64)
    args = [ctypes.byref(c)] + [None] * 7 + [0x1000, 0.125, None, None, None, 0, None]
    assert db.lib().stem_prefix_attn(*args) == sb.STEM_OK
    args[9] = 0.0
    assert db.lib().stem_prefix_attn(*args) == sb.STEM_ERR_INVALID_ARG
