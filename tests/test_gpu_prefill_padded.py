"""StemPrefill with rotary positions on a batch with rows behind its last sequence, and with sequences that are none."""
import pytest
import torch

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd.decode import Rotary
from paper_2603_06274_amd.prefill import StemPrefill

pytestmark = pytest.mark.gpu
BF, DEV = torch.bfloat16, "cuda:0"


@pytest.mark.parametrize("rotary", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_rows_behind_the_last_sequence(rotary, packed):
    g = torch.Generator().manual_seed(1)
    rows = lambda n, h: torch.randn(n, h, 64, generator=g).to(BF).to(DEV)
    n, more = 411, 29
    if packed:
        x = rows(n + more, 4)
        q, k, v = x[:, :2], x[:, 2:3], x[:, 3:]
    else:
        q, k, v = rows(n + more, 2), rows(n + more, 1), rows(n + more, 1)
    make = lambda m: StemPrefill(q[:m], k[:m], v[:m], [0, 130, n], 64, [4, 6], 1.0, n_sink=1, n_local=1,
                                 rotary=Rotary(64) if rotary else None)
    padded = make(n + more)
    padded.out.fill_(9.0)
    out = padded.run()
    assert torch.equal(out[:n], make(n).run()) and (out[n:] == 9.0).all()


def test_sequences_that_are_none():
    x = torch.zeros(100, 1, 64, dtype=BF, device=DEV)
    for cu in ([0, 60, 40], [5, 100], [0]):
        for rotary in (None, Rotary(64)):
            with pytest.raises(sb.StemError):
                StemPrefill(x, x, x, cu, 64, [2] * max(len(cu) - 1, 1), 1.0, n_sink=1, n_local=1, rotary=rotary)
    for q, k in ((x[:99], x), (x, x[:99])):
        with pytest.raises(ValueError):
            StemPrefill(q, k, k, [0, 100], 64, [2], 1.0, n_sink=1, n_local=1, rotary=Rotary(64))
