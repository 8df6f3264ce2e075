"""Tables and lse of other line lengths than the call's shape: refused, as their numbers would be taken for others'."""
import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db

from test_decode_host import P

BF = torch.bfloat16


@pytest.fixture
def host(monkeypatch):
    """Tensors of the host, and a library that says what it was called with."""
    calls = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(sb, "_raw_stream", lambda dev: P)

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or sb.STEM_OK
    monkeypatch.setattr(db, "lib", lambda: Library())
    return calls


def whole(*sizes):
    return torch.zeros(*sizes, dtype=torch.int32)


def test_block_table(host):
    shape = db.TableShape(3, 16, 20, 4, 8)
    space = torch.empty(4096, dtype=torch.uint8)
    call = lambda table: db.stem_block_table(shape, whole(3), None, whole(2), whole(20), table, whole(3), whole(2), whole(4), whole(8),
                                             whole(8), whole(4), space)
    for table in (whole(3, 5), whole(4, 3), whole(12, 1), whole(2, 4), whole(3, 8)[:, :4], whole(3, 4).t().contiguous()):
        with pytest.raises(ValueError, match="table"):
            call(table)
    assert not host
    for table in (whole(3, 4), whole(5, 4), whole(12)):
        call(table)
    assert len(host) == 3


def test_attention(host):
    q, pk = torch.zeros(3, 2, 64, dtype=BF), torch.zeros(5, 1, 64, dtype=BF)
    kp = torch.zeros(4, 16, 1, 64, dtype=BF)
    shape = db.PrefixShape.from_tensors(q, pk, db.PageShape.from_tensors(kp, kp.clone()), whole(3, 4), 1, 64)
    space = torch.empty(4096, dtype=torch.uint8)
    call = lambda table, lse: db.stem_prefix_attn(shape, q, pk, pk, kp, kp, table, whole(3), None, 0.125, torch.empty_like(q), lse, space)
    for table, lse in ((whole(3, 5), None), (whole(3, 3), None), (whole(3, 4), torch.zeros(2, 4)), (whole(3, 4), torch.zeros(3, 2))):
        with pytest.raises(ValueError):
            call(table, lse)
    assert not host
    for table, lse in ((whole(3, 4), None), (whole(12), torch.zeros(2, 3)), (whole(3, 4), torch.zeros(6))):
        call(table, lse)
    assert len(host) == 3
