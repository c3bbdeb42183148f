"""The 8-bit KV cache's host code under AddressSanitizer + UndefinedBehaviorSanitizer, on the CPU only: page table, lengths and work lists with
stand-in HIP calls and launchers that check every list against what the kernels assume (tests/sanitize/kv_san.cpp)."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import ROOT, SAN, run


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_cache_logic_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "kv_san")
    csrc = os.path.join(ROOT, "paper_2311_03285_amd", "csrc")
    src = [os.path.join(ROOT, "tests", "sanitize", "kv_san.cpp")] + [os.path.join(csrc, f) for f in ("pool.cpp", "plan.cpp", "kv8.cpp")]
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                           *src, "-o", exe])
    for seed in ("1", "2"):
        assert "kv_san OK" in run(exe, seed)
