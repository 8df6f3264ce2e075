"""The attention to a shared prefix at the ends of its range: what the host code forms of the largest sizes that it accepts (a
host-only build, launchers replaced), and what it refuses."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2603_06274_amd import binding as sb
from paper_2603_06274_amd import decode_binding as db

from test_host_sanitizers import CSRC, ROOT

NO = sb.STEM_ERR_UNSUPPORTED
MOST_SUFFIX = 2 ** 31 - 2 ** 14


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    lib = str(tmp_path_factory.mktemp("host") / "libstem_decode_host.so")
    build = ["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
             "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, *(os.path.join(CSRC, x) for x in ("stem_api.cpp", "stem_decode_api.cpp")),
             *(os.path.join(ROOT, "tests", x) for x in ("host_launch_stubs.cpp", "decode_launch_stubs.cpp", "decode_plan_stubs.cpp")),
             "-o", lib]
    res = subprocess.run(build, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return ctypes.CDLL(lib)


def shape(**kw):
    """64 requests of one token, 32 / 8 heads of 128, behind 32768 keys."""
    c = db.stem_prefix_shape(db.STEM_BF16, 32, 8, 128, 64, 64, 1, 32768, 1024, 64, 4096, 128, 1024, 128,
                             db.stem_pages(16, 4096, 16 * 1024, 1024, 128))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def plan(host, c, units=256):
    out = (ctypes.c_int64 * 10)()
    assert host.stem_test_prefix_plan(ctypes.byref(c), units, out) == sb.STEM_OK
    return dict(zip(("row_tile", "row_tiles", "prefix_splits", "split_keys", "own_tile", "own_tiles", "own_splits", "ml", "bytes", "small"),
                    list(out)))


@pytest.mark.parametrize("suffix", [2 ** 30, MOST_SUFFIX - 1, MOST_SUFFIX])
def test_the_longest_suffixes_are_split_within_32_bits(host, suffix):
    for requests in (1, 3, 15):
        c = shape(requests=requests, tokens=requests, max_suffix=suffix, pages_per_request=1 << 27)
        p = plan(host, c)
        assert 1 <= p["own_splits"] <= 64
        assert p["bytes"] < 64 * (64 + 256) * 32 * requests * 130 * 4
        for length in (1, 127, 128, suffix // 3, suffix - 1, suffix):
            keys = host.stem_test_suffix_split_keys(length, p["own_splits"])
            assert keys > 0 and keys % 128 == 0 and keys * p["own_splits"] >= length
            assert keys * p["own_splits"] < 2 ** 31 - 4 * 256      # (what a walk looks ahead)


def test_longer_suffixes_are_refused():
    n = ctypes.c_size_t()
    for suffix in (MOST_SUFFIX + 1, 2 ** 31 - 256, 2 ** 31 - 1):
        c = shape(requests=2, tokens=2, max_suffix=suffix, pages_per_request=1 << 27)
        assert db.lib().stem_prefix_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == NO


def launches(host, c, units=256):
    out = (ctypes.c_int64 * 6)()
    status = host.stem_test_prefix_launches(ctypes.byref(c), units, out)
    return status, dict(zip(("prefix_groups", "groups", "own_slots", "own_by_rows", "join_rows", "join_by_rows"), list(out)))


@pytest.mark.parametrize("requests,tokens,max_new", [(300, 8192, 8192), (256, 512, 2048), (64, 64, 4097), (64, 2111, 2048), (1, 1, 1 << 25),
                                                     (65536, 65536, 1 << 25)])
def test_launches_go_by_the_rows_that_there_are(host, requests, tokens, max_new):
    """However many new tokens a request is allowed: calls of few rows are not refused for it, and launch no more than they need."""
    c = shape(requests=requests, tokens=tokens, max_new=max_new, pages_per_request=64)
    status, l = launches(host, c)
    assert status == sb.STEM_OK
    assert l["join_rows"] <= tokens * 32
    assert l["own_slots"] <= tokens * 4 // 16 + requests
    p = plan(host, c)
    assert l["groups"] - l["prefix_groups"] == l["own_slots"] * 8 * p["own_splits"]


def test_calls_that_are_too_large_are_refused_with_their_workspace(host):
    for kw in (dict(tokens=(2 ** 31 - 1) // 32, max_new=(2 ** 31 - 1) // 32), dict(requests=65536, num_q_heads=65535, num_kv_heads=65535, tokens=1000, max_new=1, head_dim=64,
                                                      max_suffix=64, pages_per_request=4)):
        status, _ = launches(host, shape(**kw))
        assert status == NO, kw


@pytest.mark.parametrize("G,tile", [(1, 16), (4, 64), (7, 64), (3, 16), (40, 64), (1, 64)])
def test_every_row_tile_has_a_slot(host, G, tile):
    """The slots of a request's row tiles are its own, as many as it has tiles, and within those that a call has."""
    host.stem_test_slot_before.restype = ctypes.c_int64
    host.stem_test_slot_before.argtypes = [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32]
    r = random.Random(G * tile)
    for _ in range(200):
        new = [r.choice([0, 0, 1, 1, r.randint(0, 300)]) for _ in range(r.randint(1, 40))]
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        before = [host.stem_test_slot_before(x, y * G, tile) for x, y in enumerate(cu)]
        for x, n in enumerate(new):
            assert before[x + 1] - before[x] >= -(-n * G // tile) and before[x + 1] > before[x]
        # and all of them within what a call of so many tokens, and any behind them, has
        assert before[-1] <= host.stem_test_slot_before(len(new), (cu[-1] + r.randint(0, 9)) * G, tile)


@pytest.mark.parametrize("splits", [1, 2, 3, 63, 64])
def test_parts_are_counted_within_32_bits(host, splits):
    """As many as hold a key: the last of them begins before the length's end, and the next would not."""
    for length in (0, 1, 127, 128, 129, 1000, 2 ** 24 + 1, 2 ** 30, 2 ** 30 + 1, 3 * 2 ** 29, MOST_SUFFIX):
        keys, parts = host.stem_test_suffix_split_keys(length, splits), host.stem_test_suffix_parts(length, splits)
        assert parts == -(-length // keys) if length else parts == 0
        assert parts <= splits
