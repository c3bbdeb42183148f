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


def gates(dtype):
    """every 16-bit number from 2^-126 (all of binary16's) to 256, of both signs, and some beyond"""
    t = DTYPES[dtype][1]
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(t).float()
    bits = bits[(bits.abs() >= 2.0 ** -126) & (bits.abs() <= 256)]
    most = torch.finfo(t).max
    more = torch.tensor([0.0, -0.0, 1e3, -1e3, 6e4, -6e4, most, -most] + ([1e20, -1e20, 3e38, -3e38] if dtype == "bf16" else []), dtype=torch.float32).to(t)
    return torch.cat([bits.to(t), more])


@pytest.mark.parametrize("kind", [slora.ACT_SILU, slora.ACT_GELU])
@pytest.mark.parametrize("dtype,size", [("f16", s) for s in (0, 14, -20)] + [("bf16", s) for s in (0, 20, 60, 100, 120, 126, -20)])
def test_gates_of_every_size(dtype, kind, size):
    """x act(g) to 12 half-steps of fp32 (E each) before it is rounded, however small act(g) is; E are counted as: the exponential 2 and its argument's own roundings (of
    |r| <= 1, four at most, 2^-25 each times ln 2) 1.4, both once more halved in 1 + z; that sum 1, its reciprocal 2, three products 3: 3.4 + 1.7 + 1 + 2 + 3 < 12.
    x 2^n below 2^-126 is off by 2^-150 at most, times at most |g| < 2^8 where the result is not 0; g / (1 + z) between 2^-127 and 2^-126 by one half-step more.  Products of 0 and results beyond the type's range are left out."""
    lib, t = DTYPES[dtype]
    g = gates(dtype)
    width = -(-len(g) // 8) * 8
    gate = torch.zeros((2, width), dtype=t)
    gate[:, :len(g)] = g
    rng = np.random.default_rng(abs(size))
    x = (torch.from_numpy(rng.uniform(1, 2, (2, width)) * rng.choice([-1, 1], (2, width))) * 2.0 ** size).to(t)
    d_gate, d_x, y = gate.cuda(), x.cuda(), torch.empty((2, width), dtype=t, device="cuda")
    slora.w8_quantize(2, width, lib, kind, d_x.data_ptr(), width, d_gate.data_ptr(), width, y.data_ptr(), width)
    torch.cuda.synchronize()
    with np.errstate(over="ignore", invalid="ignore"):
        gd = gate.double().numpy()
        u = gd if kind == slora.ACT_SILU else 2 * np.sqrt(2 / np.pi) * (gd + 0.044715 * gd ** 3)
        ref = gd / (1 + np.exp(-u)) * x.double().numpy()
    keep = np.isfinite(ref) & (np.abs(ref) < torch.finfo(t).max * (1 - 2.0 ** -8))
    bound = 12 * du.E * np.abs(ref) + 2.0 ** -142
    du.within(y.reshape(-1)[torch.from_numpy(np.flatnonzero(keep)).cuda()], ref[keep], bound[keep])


@pytest.mark.parametrize("kind", [slora.ACT_SILU, slora.ACT_GELU])
def test_codes_of_gated_rows_are_as_close_as_fp32_allows(kind):
    """codes of rows whose gates are all -1, -5, -20, ... times x: x act(g) to 12 half-steps of fp32, so that only a code that lies so near a tie may be another"""
    width, T = 4096, 8
    x = rows(T, width, torch.float16, 4)
    gate = torch.empty_like(x)
    for t, g in enumerate([-0.01, -0.3, -1.0, -3.0, -4.5, 5.0, 20.0, 300.0]):
        gate[t] = g
    codes, scales = torch.empty((T, width), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    slora.w8_quantize(T, width, slora.F16, kind, x.data_ptr(), width, gate.data_ptr(), width, codes=codes.data_ptr(), codes_stride=width, scales=scales.data_ptr())
    torch.cuda.synchronize()
    g, v = gate.double().cpu().numpy(), x[:, :width].double().cpu().numpy()
    ref = v * g / (1 + np.exp(-(g if kind == slora.ACT_SILU else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3))))
    du.codes_within(codes, scales, ref, 12 * du.E * np.abs(ref))


@pytest.mark.parametrize("kind", [slora.ACT_SILU, slora.ACT_GELU])
@pytest.mark.parametrize("width", [1, 13, 515, 1003, 5003, 13007])
def test_what_is_behind_a_row_changes_nothing_in_it(width, kind):
    T = 6
    x, gate, out = rows(T, width, torch.bfloat16, 1, pad=8), rows(T, width, torch.bfloat16, 2, pad=8, size=2.0), []
    for behind in (0.0, float("nan"), -1e30):
        x[:, width:], gate[:, width:] = behind, behind
        y, codes, scales = torch.empty_like(x), torch.empty((T, -(-width // 16) * 16), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        slora.w8_quantize(T, width, slora.BF16, kind, x.data_ptr(), x.stride(0), gate.data_ptr(), gate.stride(0), y.data_ptr(), y.stride(0), codes.data_ptr(), codes.stride(0),
                          scales.data_ptr())
        torch.cuda.synchronize()
        out.append((y[:, :width], codes[:, :width], scales))
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))


@pytest.mark.parametrize("kind", [slora.ACT_SILU, slora.ACT_GELU])
def test_gates_below_the_normal_numbers(kind):
    """act(g) is g / 2 there, which as an fp32 number is off by 2^-150: 2^-15 of itself at most for bfloat16's least, 2^-133; x may be large"""
    g = torch.arange(1, 128, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    gate = torch.cat([g, -g, g[:2]]).reshape(1, 256).cuda()
    x, y = torch.full((1, 256), 2.0 ** 110, dtype=torch.bfloat16, device="cuda"), torch.empty((1, 256), dtype=torch.bfloat16, device="cuda")
    slora.w8_quantize(1, 256, slora.BF16, kind, x.data_ptr(), 256, gate.data_ptr(), 256, y.data_ptr(), 256)
    torch.cuda.synchronize()
    ref = gate.double().cpu().numpy() / 2 * 2.0 ** 110
    du.within(y, ref, 2.0 ** -15 * np.abs(ref))
