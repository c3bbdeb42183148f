"""Wavefronts that the kernels' comments count on, from the compiler's own report of registers (no GPU needed): two workgroups of prompts and three of few columns
share a compute unit up to heads of 128 elements, three of the shared-x product do with one tile of outputs."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2311_03285_amd import build as hip_build

pytestmark = pytest.mark.skipif(shutil.which(hip_build.HIPCC) is None and not os.path.exists(hip_build.HIPCC), reason="no hipcc")


def occupancy(source, tmp_path):
    """of each kernel: wavefronts a SIMD by registers and static LDS"""
    r = subprocess.run([hip_build.HIPCC] + hip_build.FLAGS + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, source), "-o", str(tmp_path / "k.s"),
                                                              "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    found, name = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"remark: Function Name: (\S+)", line)
        name = m.group(1) if m else name
        m = re.search(r"remark:\s+Occupancy \[waves/SIMD\]: (\d+)", line)
        if m and name:
            found[name] = int(m.group(1))
    return found


def test_attention(tmp_path):
    found = occupancy("kv8_kernels.hip", tmp_path)
    seen = 0
    for name, waves in found.items():
        m = re.search(r"kv_attend_(few|many)_kernelILi[01]ELi(\d)E", name)
        if m:
            seen += 1
            least = {"few": 3 if int(m.group(2)) <= 4 else 2 if m.group(2) == "6" else 1, "many": 2 if int(m.group(2)) <= 4 else 1}[m.group(1)]
            assert waves >= least, (name, waves)
    assert seen == 24


def test_4_bit_products(tmp_path):
    found = occupancy("w4_kernels.hip", tmp_path)
    seen = 0
    for name, waves in found.items():
        m = re.search(r"w4_wide_kernelILi[01]ELi(\d)ELi(\d)ELi(\d)ELi(\d+)E", name)
        if m:
            teams, tiles, tokens, unit = map(int, m.groups())
            seen += 1
            assert waves >= (6 if teams == 2 and tiles == 1 and tokens <= 2 and (unit > 32 or tokens == 1) else 2), (name, waves)
    assert seen > 20
