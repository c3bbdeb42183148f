"""Products whose sum times x's scale leaves fp32's range, though y does not: rows of bfloat16 up to 3e38 have such scales."""
import numpy as np
import pytest
import torch

from dense_util import product, within
from paper_2311_03285_amd import slora
from test_gpu_w8 import Matrix, X, run

pytestmark = pytest.mark.gpu


def matrix(outputs, inputs, seed, scales):
    """... with scales of one's own behind the packed codes, 16 to a tile"""
    m = Matrix(outputs, inputs, seed, "bf16")
    m.scales = scales.astype(np.float32)
    at = slora.w8_bytes(outputs, inputs) // 4 - -(-outputs // 16) * 16
    m.packed.view(torch.float32)[at:at + outputs].copy_(torch.from_numpy(m.scales))
    return m


def mixed(T, inputs, seed, sizes):
    """rows whose scales are of the given sizes in turn"""
    x = X(T, inputs, seed)
    x.scales = (x.scales * 70 * 2.0 ** np.resize(np.asarray(sizes, float), T)).astype(np.float32)
    x.d_scales.copy_(torch.from_numpy(x.scales))
    return x


@pytest.mark.parametrize("y16", [False, True])
@pytest.mark.parametrize("T", [1, 5, 16, 40, 70, 200, 300, 513])
def test_large_scales_of_x(T, y16):
    """2^90 .. 2^121 beside ordinary ones, weights' scales of 2^-60 and 2^-126: a sum of up to 2^23 passes 2^128 on the way"""
    rng = np.random.default_rng(T)
    sizes = [100, -7, 112, 121, 90, 0]
    for w_size in (-60, -126):
        m, x = matrix(300, 520, 3, rng.uniform(0.5, 1, 300) * 2.0 ** w_size), mixed(T, 520, 4, sizes)
        ref, bound = product(x.codes, x.scales, m.codes, m.scales)
        assert np.abs(ref).max() < 2.0 ** 127
        within(run([m], [x], T, y16)[0], ref, bound + 2.0 ** -149)


@pytest.mark.parametrize("T", [3, 90])
def test_scales_that_cancel_give_the_same_bits(T):
    """the ranges of the two scales are powers of two apart, so that only they may differ"""
    x, base = mixed(T, 260, 5, [0]), np.random.default_rng(1).uniform(0.5, 1, 100)
    m = matrix(100, 260, 6, base)
    want = run([m], [x], T, False)[0].clone()
    for size in (-100, 64, 95, 96, 97, 110, 120):
        x2, m2 = mixed(T, 260, 5, [size]), matrix(100, 260, 6, base * 2.0 ** -size)
        assert torch.equal(run([m2], [x2], T, False)[0], want), size


@pytest.mark.parametrize("T", [2, 50])
def test_sums_of_0_and_spoiled_rows(T):
    m = matrix(40, 64, 7, np.full(40, 2.0 ** 100))
    x = mixed(T, 64, 8, [120])
    x.d_codes.zero_()
    assert (run([m], [x], T, False)[0] == 0).all()
    x = mixed(T, 64, 8, [120])
    x.d_scales[0], x.d_scales[1] = float("inf"), float("nan")
    y = run([m], [x], T, False)[0]
    assert not torch.isfinite(y[0]).any() and torch.isnan(y[1]).all()
    x = mixed(T, 64, 8, [120])
    x.d_scales.neg_()
    m = matrix(40, 64, 7, np.full(40, 2.0 ** -60))
    ref, bound = product(x.codes, -x.scales, m.codes, m.scales)
    within(run([m], [x], T, False)[0], ref, bound)


def test_a_large_row_from_its_values_to_y():
    """bfloat16 values of 3e38 in 8 bits, times weights of 2^-12"""
    n, O = 512, 64
    rng = np.random.default_rng(2)
    v = torch.from_numpy(rng.uniform(0.5, 1, (20, n)) * 2.0 ** 127).bfloat16().cuda()
    codes, scales = torch.empty((20, n), dtype=torch.int8, device="cuda"), torch.empty(20, device="cuda")
    m = matrix(O, n, 9, rng.uniform(0.5, 1, O) * 2.0 ** -27)
    for T in (4, 20):
        slora.w8_quantize(T, n, slora.BF16, slora.ACT_NONE, v.data_ptr(), n, codes=codes.data_ptr(), codes_stride=n, scales=scales.data_ptr())
        y = torch.empty((T, O), device="cuda")
        slora.w8_matmul([m.handle], [codes.data_ptr()], [n], [scales.data_ptr()], T, [y.data_ptr()], [O])
        torch.cuda.synchronize()
        ref, bound = product(codes[:T].cpu().numpy(), scales[:T].cpu().numpy(), m.codes, m.scales)
        within(y, ref, bound)
        assert np.abs(ref).max() < 2.0 ** 127
