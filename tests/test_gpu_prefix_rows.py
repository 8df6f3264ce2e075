"""stem_prefix_attn where requests are allowed many more new tokens than they have: row tiles and joined rows are counted by the rows that
there are, and their requests are looked up in cu_new."""
import pytest
import torch

from test_gpu_prefix_attn import BF, HF, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,dtype", [(8, 2, 64, BF), (8, 1, 128, HF), (2, 2, 256, BF), (1, 1, 128, BF)])
@pytest.mark.parametrize("L", [0, 20, 900])            # few parts and many
def test_a_prompt_beside_single_tokens(Hq, Hkv, d, dtype, L):
    new = [1] * 20 + [0, 0, 301, 0] + [1, 3] * 9 + [0]
    c = Case([(37 * i) % 90 for i in range(len(new))], new, L, Hq, Hkv, d, 16, dtype, padding=7, seed=L + d)
    for c.max_new in (301, 2048, 1 << 20):
        c.check(*c.run())


@pytest.mark.parametrize("R", [64, 65, 130, 5000])     # one load of 64 entries, two, three
def test_requests_are_found(R):
    new = [(i * 7) % 3 if i % 64 else 0 for i in range(R)]
    new[-1], new[R // 2] = 0, 40
    c = Case([i % 5 for i in range(R)], new, 30, 2, 1, 64, 16, padding=3, seed=R)
    c.max_new = 1000
    c.check(*c.run())


def test_rows_beyond_the_promised_are_left():
    new = [0] * 30
    new[3], new[4], new[20] = 50, 7, 21
    c = Case([9] * 30, new, 200, 8, 2, 64, padding=5, seed=3)
    c.max_new = 20
    out, z = c.run()
    c.check(out, z)
    assert (out[20:50] == 9.0).all() and (out[77:78] == 9.0).all() and not (out[50:57] == 9.0).any()


def test_one_token_each_whatever_is_allowed():
    c = Case([300 * (i % 2) for i in range(70)], [1] * 70, 500, 8, 2, 64, seed=4)
    c.max_new = 500
    a, b = c.run(), c.run(use_cu=False, lse=False)
    c.check(*a)
    assert torch.equal(a[0], b[0])


def test_few_rows_are_not_refused_for_a_large_bound():
    c = Case([40] * 64, [1] * 64, 2048, 32, 8, 64, seed=5)
    c.max_new = 4097
    c.check(*c.run())
