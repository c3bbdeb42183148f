"""Resources of the kernels of norms, rows in 8 bits and products with 8-bit weights, from the compiler's own report (no GPU needed): no spilled registers, no
scratch memory, no packed-fp32 instructions, and as many wavefronts as the kernels' comments count on."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2311_03285_amd import build as hip_build
from test_kernel_occupancy_attention import occupancy

pytestmark = pytest.mark.skipif(shutil.which(hip_build.HIPCC) is None and not os.path.exists(hip_build.HIPCC), reason="no hipcc")


@pytest.mark.parametrize("source,least", [("rows_kernels.hip", 40), ("w8_kernels.hip", 34)])
def test_no_kernel_spills_or_uses_scratch(source, least, tmp_path):
    asm = str(tmp_path / "k.s")
    r = subprocess.run([hip_build.HIPCC] + hip_build.FLAGS + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, source), "-o", asm,
                                                              "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    name, kernels = None, set()
    for line in r.stderr.splitlines():
        m = re.search(r"remark: Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            kernels.add(name)
        m = re.search(r"remark:\s+(ScratchSize|VGPRs Spill|SGPRs Spill)(?: \[[^\]]*\])?: (\d+)", line)
        if m:
            assert int(m.group(2)) == 0, (name, line)
    assert len(kernels) >= least
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", open(asm).read())


def test_wavefronts(tmp_path):
    """16 wavefronts of a row fit a compute unit; products of 256 x 256 and 256 x 192 have two wavefronts a SIMD, the smaller ones three workgroups' or more"""
    for name, waves in occupancy("rows_kernels.hip", tmp_path).items():
        assert waves >= 4, (name, waves)
    seen = 0
    for name, waves in occupancy("w8_kernels.hip", tmp_path).items():
        m = re.search(r"w8_tile_kernelILi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELb[01]E", name)
        if m:
            seen += 1
            assert waves >= (2 if int(m.group(4)) * int(m.group(5)) >= 6 else 3), (name, waves)
    assert seen == 48
