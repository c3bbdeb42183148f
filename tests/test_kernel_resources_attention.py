"""Resources of the kernels of the 8-bit KV cache and the 4-bit products, from the compiler's own report (no GPU needed): no spilled
registers, no scratch memory, no packed-fp32 instructions, and as many wavefronts as the kernels' comments count on."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2311_03285_amd import build as hip_build

pytestmark = pytest.mark.skipif(shutil.which(hip_build.HIPCC) is None and not os.path.exists(hip_build.HIPCC), reason="no hipcc")


@pytest.fixture(scope="module", params=["kv8_kernels.hip", "w4_kernels.hip"])
def report(request, tmp_path_factory):
    asm = str(tmp_path_factory.mktemp("res") / "k.s")
    r = subprocess.run([hip_build.HIPCC] + hip_build.FLAGS + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, request.param), "-o", asm,
                                                              "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    kernels, name = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"remark: Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            kernels[name] = {}
            continue
        m = re.search(r"remark:\s+([A-Za-z ]+?)(?: \[[^\]]*\])?: (\d+)", line)
        if m and name:
            kernels[name][m.group(1).strip()] = int(m.group(2))
    return kernels, open(asm).read()


def test_no_kernel_spills_or_uses_scratch(report):
    kernels, asm = report
    assert len(kernels) >= 15
    for k, v in kernels.items():
        assert v.get("ScratchSize", 0) == 0 and v.get("VGPRs Spill", 0) == 0 and v.get("SGPRs Spill", 0) == 0, (k, v)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)
