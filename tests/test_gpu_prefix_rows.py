"""stem_prefix_attn where requests are allowed many more new tokens than they have: row tiles and joined rows are counted by the rows that
there are, and their requests are looked up in cu_new."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db

import decode_util as du
from test_gpu_prefix_attn import BF, DEV, HF, Case

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


def test_launches_of_more_than_one_line():
    """65536 requests of 32 KV heads: 2^21 workgroups of own keys.  (Their pages are shared, which reading does not mind.)"""
    R, H, d, N, L = 65536, 32, 64, 300, 20
    g = torch.Generator(device=DEV).manual_seed(9)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV).to(BF)
    q, pk, pv, kp, vp = normal(R, H, d), normal(L, H, d), normal(L, H, d), normal(N, 16, H, d), normal(N, 16, H, d)
    table = torch.randint(0, N, (R, 1), generator=g, device=DEV, dtype=torch.int32)
    lens = torch.randint(1, 7, (R,), generator=g, device=DEV, dtype=torch.int32)
    shape = db.PrefixShape.from_tensors(q, pk, db.PageShape.from_tensors(kp, vp), table, 1, 16)
    space = torch.full((db.stem_prefix_attn_workspace_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, 9.0)
    db.stem_prefix_attn(shape, q, pk, pv, kp, vp, table, lens, None, d ** -0.5, out, None, space)
    assert not (out == 9.0).all(dim=2).any() and out.isfinite().all()
    line = 2 ** 20 // H                                # requests of the first line
    some = [0, 1, 7, 8, line - 9, line - 2, line - 1, line, line + 1, line + 8, R - 9, R - 2, R - 1, *range(100, R, 3001)]
    for r in some:
        k, v = (torch.cat([x, p[table[r, 0], :lens[r]]]).cpu().double() for x, p in ((pk, kp), (pv, vp)))
        o, bound, _, _ = du.attention_rows(q[r].cpu().double(), k, v, d ** -0.5, BF)
        assert ((out[r].cpu().double() - o).abs() <= bound).all(), r
