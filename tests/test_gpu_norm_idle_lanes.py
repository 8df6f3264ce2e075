"""Heads of fewer values than their lanes have room for, whose halves are exchanged between lanes: lanes without values take no part."""
import pytest

from test_gpu_norm_odd_halves import BF, FP, HF, test_new_tokens as new_tokens, test_values_and_gradients as values_and_gradients

pytestmark = pytest.mark.gpu
SIZES = [(24, 18), (32, 26), (32, 30), (40, 38), (72, 42), (72, 70), (96, 82), (136, 134), (200, 130), (264, 262), (520, 518), (776, 2)]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("d,rot", SIZES)
def test_values_and_gradients(dtype, d, rot):
    values_and_gradients(dtype, d, rot)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rot", SIZES)
def test_new_tokens(dtype, d, rot):
    new_tokens(dtype, d, rot)
