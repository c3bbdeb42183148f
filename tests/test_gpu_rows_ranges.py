"""Norms and gates where 32-bit steps come to the ends of their range: what the formulas give there is still the result."""
import numpy as np
import pytest
import torch

import dense_util as du
from paper_2311_03285_amd import slora
from test_gpu_rows import DTYPES, Norm, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h32", [False, True])
@pytest.mark.parametrize("width", [1, 40, 512, 700, 4096, 17000, 32768])
def test_layer_norms_of_equal_values_are_the_bias(width, h32):
    """v - mean is 0 whatever v is, and so is its quotient by the root of eps.  Sums of a power of two are exact, so that 0 is; sums of 2^120 leave the range."""
    for eps in (2.0 ** -60, 1e-5, 3.0):
        m = Norm(width, "bf16", layer=True, bias=True, h32=h32, eps=eps, seed=width)
        h = torch.zeros((7, -(-width // 8) * 8), dtype=torch.float32 if h32 else torch.bfloat16, device="cuda")
        for t, v in enumerate((0.0, 2.0 ** -120, 1.0, -(2.0 ** 100), 2.0 ** 110, 2.0 ** 120, -(2.0 ** 127))):
            h[t] = v
        out = m(h)
        bias = m.pre[1]
        assert torch.equal(out["x"], bias.expand(7, width))
        codes, scales = du.codes_of(bias.float().cpu().numpy()[None])
        assert np.array_equal(out["codes"].cpu().numpy(), np.repeat(codes, 7, axis=0)) and np.array_equal(out["scales"].cpu().numpy(), np.repeat(scales, 7))


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("width", [64, 700, 4096])
def test_an_eps_above_every_square(width, layer):
    """rows of 2^-40 .. 2^70 with an eps of 2^110: quotients are small numbers, not 0"""
    m = Norm(width, "bf16", layer=layer, eps=2.0 ** 110)
    h = rows(4, width, torch.bfloat16, 1)
    for t, e in enumerate([-40, -10, 20, 70]):
        h[t, :width] = h[t, :width] * 2.0 ** e
    m.check(h)


@pytest.mark.parametrize("layer", [False, True])
def test_large_rows_with_an_eps(layer):
    """2^20 .. 2^120: squares leave the range, and eps is nothing beside them"""
    for width in (64, 700, 4096, 17000):
        m = Norm(width, "bf16", layer=layer, post=True, bias=True, eps=1e-5)
        h = rows(5, width, torch.bfloat16, 1)
        for t, e in enumerate([20, 60, 80, 110, 120]):
            h[t, :width] = h[t, :width] * 2.0 ** e
        m.check(h)
        m.check(rows(5, width, torch.bfloat16, 2), h)
