"""The C-ABI front ends of moa_rope.h and moa_kv4.h under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): built for the host with both, their kernel launchers replaced
by stand-ins that report no device, and run through tests/test_rope_kv4_api.py."""
import os
import subprocess
import sys

import pytest

from test_sanitizers import CSRC, ROOT, SAN_FLAGS, _run


def test_rope_and_kv4_api_under_sanitizers(tmp_path):
    if not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("HIP headers not installed")
    if not os.path.exists(os.path.join(ROOT, "paper_2606_07713_amd", "libmoa_attn.so")):
        pytest.skip("HIP library not built (the binding needs it to import)")
    lib = str(tmp_path / "libmoa_attn_san.so")
    stubs = [os.path.join(ROOT, "tests", "sanitize", f) for f in ("launch_stub.cpp", "rope_kv4_stub.cpp")]
    _run(["g++", "-std=c++17", *SAN_FLAGS, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
          *[os.path.join(CSRC, f) for f in ("api.cpp", "api_rope.cpp", "api_kv4.cpp")], *stubs,
          "-o", lib, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    asan = subprocess.run(["gcc", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", MOA_TEST_SANITIZED_API_LIB=lib)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        "tests/test_rope_kv4_api.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error:" not in r.stderr, tail
    assert " passed" in r.stdout, tail
