"""The host code of include/stem_decode.h built for the CPU only with AddressSanitizer and UndefinedBehaviorSanitizer, the kernel
launchers replaced by no-op stand-ins (tests/decode_launch_stubs.cpp), and its host tests run against that build in a child process."""
import os
import shutil
import subprocess
import sys

import pytest

from test_host_sanitizers import CSRC, ROOT, _runtime


@pytest.mark.skipif(shutil.which("g++") is None or _runtime("libasan.so") is None or _runtime("libubsan.so") is None
                    or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"),
                    reason="needs g++ with the ASan/UBSan runtimes and the HIP headers")
def test_decode_host_code_under_address_and_ub_sanitizers(tmp_path):
    lib = str(tmp_path / "libstem_decode_host_san.so")
    build = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-fno-omit-frame-pointer",
             "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
             "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
             *(os.path.join(CSRC, x) for x in ("stem_api.cpp", "stem_decode_api.cpp")),
             *(os.path.join(ROOT, "tests", x) for x in ("host_launch_stubs.cpp", "decode_launch_stubs.cpp")), "-o", lib]
    res = subprocess.run(build, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    preload = [_runtime("libasan.so"), _runtime("libubsan.so")]
    if os.environ.get("LD_PRELOAD"):
        preload.append(os.environ["LD_PRELOAD"])
    env = dict(os.environ, LD_PRELOAD=":".join(preload), STEM_HIP_LIBRARY=lib,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               PYTHONDONTWRITEBYTECODE="1")
    run = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_decode_host.py"), "-x", "-q",
                          "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True)
    assert run.returncode == 0, (run.stdout[-3000:], run.stderr[-3000:])
    assert "passed" in run.stdout and "skipped" not in run.stdout
    assert "Sanitizer" not in run.stderr and "runtime error" not in run.stderr
