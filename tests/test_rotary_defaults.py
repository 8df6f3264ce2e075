"""The numbers of turns that a scaling method begins and ends at when none are given: those of the method."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd.decode import Rotary

from test_decode_host import plain_frequencies


@pytest.mark.parametrize("kind,high", [("none", 4.0), ("linear", 4.0), ("ntk", 4.0), ("yarn", 32.0), ("bands", 4.0)])
def test_turns_by_default(kind, high):
    given, f0 = db.stem_rotary_frequencies(128, 10000.0, kind, 8.0, 4096.0, 1.0, high)
    default, f1 = db.stem_rotary_frequencies(128, 10000.0, kind, 8.0, 4096.0)
    rotary = Rotary(128, theta=10000.0, scaling=kind, factor=8.0, trained_length=4096.0, device="cpu")
    assert torch.equal(given, default) and torch.equal(given, rotary.turns) and f0 == f1 == rotary.attention_factor
    want = torch.tensor(plain_frequencies(128, 10000.0, kind, 8.0, 4096.0, 1.0, high), dtype=torch.float64) / (2 * torch.pi)
    assert ((default - want).abs() <= 1e-13 * want).all()


def test_given_turns_are_taken():
    four, _ = db.stem_rotary_frequencies(128, 10000.0, "yarn", 8.0, 4096.0, 1.0, 4.0)
    more, _ = db.stem_rotary_frequencies(128, 10000.0, "yarn", 8.0, 4096.0)
    assert not torch.equal(four, more)
