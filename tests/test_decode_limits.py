"""The attention to a shared prefix at the ends of its range: what the host code forms of the largest sizes that it accepts (a
host-only build, launchers replaced), and what it refuses."""
import ctypes
import os
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
