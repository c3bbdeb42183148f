"""The sizes by which the GPU tests mean to run every shape of tiles do so by the library's own rule, compiled for the host; and the rule for loads of weights without a
place in the caches."""
import os
import shutil
import subprocess

import pytest

from test_gpu_w8 import SHAPES
from test_host_sanitizers import ROOT, SAN, run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    exe, csrc = str(tmp_path_factory.mktemp("shapes") / "w8_shapes"), os.path.join(ROOT, "paper_2311_03285_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                           os.path.join(ROOT, "tests", "sanitize", "w8_shapes.cpp"), os.path.join(csrc, "w8.cpp"), "-o", exe])

    def ask(calls):
        """of (matrices, outputs, inputs, tokens): ((outputs, tokens) of a tile, once)"""
        *lines, last = run(exe, *(str(v) for c in calls for v in c)).splitlines()
        assert last == f"{len(SHAPES)} shapes"
        found = [tuple(int(v) for v in line.split()) for line in lines]
        return [(f[:2], bool(f[2])) for f in found]

    return ask


def test_every_shape_is_taken(answers):
    calls, want = [], []
    for shape, (outputs, T) in SHAPES.items():
        for o in (outputs, outputs // 8 * 8, outputs // 8 * 8 + 3):  # as test_every_shape_of_tiles and test_weights_too_large_for_the_caches have them
            calls.append((1, o, 390, T))
            want.append((shape, False))
    assert answers(calls) == want


def test_both_loads_of_weights(answers):
    """weights too large for the caches: those of calls of one round, or of one tile of tokens, are loaded without a place there, and only those"""
    calls = [(1, outputs, -(-(68 << 20) // outputs), T) for outputs, T in SHAPES.values()]
    took = answers(calls)
    assert [s for s, _ in took] == list(SHAPES)
    assert {s for s, once in took if once} >= set(list(SHAPES)[2:])  # the shapes that have both
    assert [once for _, once in answers([(2, 20480, 5120, 32), (2, 20480, 5120, 100), (4, 4096, 4096, 512), (3, 4096, 4096, 24), (2, 20480, 5120, 200), (2, 20480, 5120, 900)])] == [
        True, True, True, False, False, False]
