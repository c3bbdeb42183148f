"""Norms, rows in 8 bits and products with 8-bit weights without a GPU: every refusal, and what their kernels assume of their arguments, under
AddressSanitizer + UndefinedBehaviorSanitizer (tests/sanitize/dense_san.cpp); the binding; the helpers that the GPU tests go by."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import dense_util as du
from paper_2311_03285_amd import slora
from test_host_sanitizers import ROOT, SAN, run


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_refusals_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "dense_san")
    csrc = os.path.join(ROOT, "paper_2311_03285_amd", "csrc")
    src = [os.path.join(ROOT, "tests", "sanitize", "dense_san.cpp")] + [os.path.join(csrc, f) for f in ("rows.cpp", "w8.cpp")]
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                           *src, "-o", exe])
    assert "dense_san OK" in run(exe)


def test_the_binding_passes_on_what_the_library_refuses():
    for call in (lambda: slora.norm_init(0, slora.F16), lambda: slora.norm_init(64, slora.F16, eps=-1.0), lambda: slora.w8_bytes(0, 5), lambda: slora.w8_bytes(5, 131072),
                 lambda: slora.w8_pack(5, 5, 7, 16, 16, 16), lambda: slora.w8_quantize(2, 64, slora.F16, slora.ACT_SILU, 16, 64, y=32, y_stride=64),
                 lambda: slora.norm_apply(None, 1, 16, 64)):
        with pytest.raises(slora.SloraError) as e:
            call()
        assert e.value.code == slora.EINVAL
    for call in (slora.w8_matmul, slora.w8_matmul_y16):
        with pytest.raises(ValueError):
            call([None], [16, 32], [16], [16], 1, [16], [16])
        with pytest.raises(slora.SloraError, match="is NULL"):
            call([None], [16], [16], [16], 1, [16], [16])
    slora.w8_quantize(0, 64, slora.F16, slora.ACT_NONE, 0, 0)
    assert slora.w8_bytes(16, 128) == 2 * 1024 + 64


def test_rows_in_8_bits_by_the_definition():
    v = np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5], [0, 0, 0, 0, 0, 0], [1e-35, 0, 0, 0, 0, 0], [np.inf, 1, 2, 3, 4, 5], [np.nan, 1, 2, 3, 4, 5]], np.float32)
    c, s = du.codes_of(v)
    assert c[0].tolist() == [127, 0, 2, 2, 0, -2] and s[0] == 1.0
    assert (c[1:] == 0).all() and s[1] == s[2] == np.float32(2.0 ** -100) / np.float32(127) and np.isnan(s[3:]).all()


def test_norms_and_their_bounds_by_a_plain_evaluation_in_32_bits():
    """what the bounds allow holds of torch's fp32, and a mistake of one part in 10^4 does not"""
    rng = np.random.default_rng(0)
    h, b = rng.standard_normal((3, 700)) * 3, rng.standard_normal((3, 700))
    w, c = 1 + 0.2 * rng.standard_normal(700), 0.2 * rng.standard_normal(700)
    h, b, w, c = (torch.from_numpy(a).half() for a in (h, b, w, c))
    d = [a.double().numpy() for a in (h, b, w, c)]
    for layer in (False, True):
        h2, eh, x, ex = du.norm(d[0], d[1], None, 0.5, (d[2], d[3]), (d[2], d[3]), layer, 1e-5)

        def plain(v):
            if layer:
                v = v - v.mean(dim=1, keepdim=True)
            return v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + 1e-5) * w.float() + c.float()

        got = h.float() + 0.5 * plain(b.float())
        du.within(got, h2, eh)
        du.within(plain(got), x, ex)
        with pytest.raises(AssertionError):
            du.within(plain(got) * (1 + 1e-4), x, ex)
        assert (eh < 1e-4 * (1 + np.abs(h2))).all() and (ex < 1e-4 * (1 + np.abs(x))).all()
