"""What orders the wavefronts of an eviction's selection in LDS, checked on the CPU (tests/sanitize/evict_turns.cpp)."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import ROOT, SAN, run


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_no_array_of_bins_is_cleared_while_another_wavefront_may_read_it(tmp_path):
    exe = str(tmp_path / "evict_turns")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
                           "-I" + os.path.join(ROOT, "paper_2311_03285_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize", "evict_turns.cpp"), "-o", exe])
    assert "evict_turns OK" in run(exe)
