"""The largest sizes of test_memory_limits_host.py, planned by host code under AddressSanitizer and UndefinedBehaviorSanitizer (CPU)."""
import glob
import os
import subprocess
import sys

import pytest

from conftest import ROOT


def test_host_side_under_asan_and_ubsan():
    lib = os.path.join(ROOT, "paper_2604_12841_amd", "libpredecoder_san.so")
    if not os.path.exists(lib):
        pytest.skip("libpredecoder_san.so not built (python paper_2604_12841_amd/build.py --sanitize)")
    rt = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    if not rt:
        pytest.skip("no clang AddressSanitizer runtime")
    env = dict(os.environ, LD_PRELOAD=rt[0], ASAN_OPTIONS="detect_leaks=0", PD_LIBRARY=lib, UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu",
                        os.path.join(ROOT, "tests", "test_memory_limits_host.py")], capture_output=True, text=True, env=env, cwd=ROOT, timeout=900)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]
