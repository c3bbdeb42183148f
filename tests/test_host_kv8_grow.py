"""How an 8-bit cache's page lists grow (tests/sanitize/kv_grow.cpp): without copying the whole list for each block."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import ROOT, SAN, run


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_a_list_that_grows_by_blocks_is_not_copied_for_each(tmp_path):
    exe = str(tmp_path / "kv_grow")
    csrc = os.path.join(ROOT, "paper_2311_03285_amd", "csrc")
    src = [os.path.join(ROOT, "tests", "sanitize", "kv_grow.cpp")] + [os.path.join(csrc, f) for f in ("pool.cpp", "plan.cpp", "kv8.cpp")]
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                           *src, "-o", exe])
    assert "kv_grow OK" in run(exe)
