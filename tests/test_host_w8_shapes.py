"""The sizes by which the GPU tests mean to run every shape of tiles do so by the library's own rule, compiled for the host."""
import os
import shutil
import subprocess

import pytest

from test_gpu_w8 import SHAPES
from test_host_sanitizers import ROOT, SAN, run


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_every_shape_is_taken(tmp_path):
    exe, csrc = str(tmp_path / "w8_shapes"), os.path.join(ROOT, "paper_2311_03285_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                           os.path.join(ROOT, "tests", "sanitize", "w8_shapes.cpp"), os.path.join(csrc, "w8.cpp"), "-o", exe])
    sizes = []
    for outputs, T in SHAPES.values():
        for o in (outputs, outputs // 8 * 8, outputs // 8 * 8 + 3):  # as test_every_shape_of_tiles and test_weights_too_large_for_the_caches have them
            sizes += [o, T]
    *lines, last = run(exe, *map(str, sizes)).splitlines()
    want = [f"{o} {t}" for o, t in SHAPES for _ in range(3)]
    assert lines == want and last == f"{len(SHAPES)} shapes"
