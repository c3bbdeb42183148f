"""GPU parity of the products with 4-bit weights against numpy in 64 bits; the bound is that of an fp32 sum of the products of c and
of z (np_kv8.w4), plus one rounding for a 16-bit y."""
import numpy as np
import pytest
import torch

from oracle import np_kv8
from paper_2311_03285_amd import slora

pytestmark = pytest.mark.gpu
DTYPES = {"f16": (slora.F16, torch.float16), "bf16": (slora.BF16, torch.bfloat16)}


class Matrix:
    def __init__(self, outputs, inputs, group, dtype, zeros, seed):
        rng = np.random.default_rng(seed)
        groups = -(-inputs // group)
        self.lib_dtype, t = DTYPES[dtype]
        self.shape, self.group = (outputs, inputs), group
        self.codes = rng.integers(0, 16, (outputs, inputs), dtype=np.uint8)
        scales = torch.from_numpy(rng.uniform(0.5, 1.5, (outputs, groups)) / 4.6 / inputs ** 0.5).to(t)
        self.scales = scales.double().numpy()
        self.zeros = rng.integers(0, 16, (outputs, groups), dtype=np.uint8) if zeros else np.full((outputs, groups), 8, np.uint8)
        d_codes = torch.from_numpy(self.codes[:, 0::2] | (self.codes[:, 1::2] << 4)).cuda()
        d_scales, d_zeros = scales.cuda(), torch.from_numpy(self.zeros).cuda()
        self.packed = torch.full((slora.w4_bytes(outputs, inputs, group),), 0xA5, dtype=torch.uint8, device="cuda")
        self.handle = slora.w4_pack(outputs, inputs, group, self.lib_dtype, d_codes.data_ptr(), d_scales.data_ptr(),
                                    d_zeros.data_ptr() if zeros else None, self.packed.data_ptr())
        torch.cuda.synchronize()

    def reference(self, x):
        return np_kv8.w4(x.double().cpu().numpy(), self.codes, self.scales, self.zeros, self.group)


def run(ms, xs, T, y16, stream=None):
    t = xs[0].dtype
    guard = [torch.full((T + 1, m.shape[0]), 7.0, dtype=t if y16 else torch.float32, device="cuda") for m in ms]
    torch.cuda.synchronize()
    (slora.w4_matmul_y16 if y16 else slora.w4_matmul)([m.handle for m in ms], [x.data_ptr() for x in xs], T, [y.data_ptr() for y in guard], stream)
    torch.cuda.synchronize()
    for y in guard:
        assert (y[T] == 7.0).all()
    return [y[:T] for y in guard]


def check(ms, xs, ys):
    for m, x, y in zip(ms, xs, ys):
        ref, bound = m.reference(x[:len(y)])
        half = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[y.dtype]
        err = np.abs(y.double().cpu().numpy() - ref)
        assert (err <= bound + np.abs(ref) * half + 2.0 ** -24 * (half > 0)).all(), float((err - bound).max())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("y16", [False, True])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 32, 33, 48, 64, 65, 130, 257])
def test_tokens(T, dtype, y16):
    ms = [Matrix(200, 520, 128, dtype, True, 1), Matrix(33, 520, 128, dtype, False, 2)]
    x = torch.randn(T, 520, device="cuda").to(DTYPES[dtype][1])
    check(ms, [x, x], run(ms, [x, x], T, y16))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 160, 256, 1 << 20])
@pytest.mark.parametrize("outputs,inputs", [(1, 8), (16, 128), (17, 136), (5, 1000), (70, 3080), (256, 4096)])
def test_shapes_and_groups(outputs, inputs, group, dtype):
    for T in (1, 20, 70):
        m = Matrix(outputs, inputs, group, dtype, True, outputs + group)
        x = torch.randn(T, inputs, device="cuda").to(DTYPES[dtype][1])
        check([m], [x], run([m], [x], T, False))


def test_eight_matrices_of_different_shapes():
    ms = [Matrix(o, i, 64, "bf16", o % 2 == 0, o) for o, i in [(16, 64), (100, 8), (3, 2048), (512, 512), (31, 136), (64, 64), (1, 1000), (40, 320)]]
    xs = [torch.randn(9, m.shape[1], device="cuda").bfloat16() for m in ms]
    check(ms, xs, run(ms, xs, 9, False, torch.cuda.Stream()))


def test_every_code_times_every_place():
    """one input at a time: each weight by itself, exactly"""
    for dtype in ("f16", "bf16"):
        m = Matrix(64, 256, 32, dtype, True, 5)
        x = torch.eye(256, device="cuda").to(DTYPES[dtype][1])
        y = run([m], [x], 256, False)[0].double().cpu().numpy()
        g = np.arange(256) // 32
        w = (m.codes.astype(np.float64) - m.zeros[:, g]) * m.scales[:, g]
        assert np.array_equal(y, w.T)  # few bits times few bits: no rounding


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_and_offset_activations(dtype):
    m = Matrix(96, 2048, 128, dtype, False, 9)
    x = torch.randn(5, 2048, device="cuda") + 10.0
    x[:, 7] = 3000.0
    x = x.to(DTYPES[dtype][1])
    check([m], [x], run([m], [x], 5, False))


def test_an_infinite_token_leaves_the_others_alone():
    m = Matrix(50, 300 // 8 * 8, 64, "f16", True, 4)
    x = torch.randn(20, m.shape[1], device="cuda").half()
    clean = run([m], [x], 20, False)[0]
    x2 = x.clone()
    x2[3, 100], x2[17, 0] = float("inf"), float("nan")
    y = run([m], [x2], 20, False)[0]
    others = [t for t in range(20) if t not in (3, 17)]
    assert torch.equal(y[others], clean[others]) and not torch.isfinite(y[3]).all() and torch.isnan(y[17]).all()


def test_a_graph_replays_the_product():
    m = Matrix(128, 1024, 128, "bf16", False, 3)
    x = torch.zeros(4, 1024, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(4, 128, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        slora.w4_matmul([m.handle], [x.data_ptr()], 4, [y.data_ptr()], torch.cuda.current_stream())
    for _ in range(3):
        x.copy_(torch.randn(4, 1024))
        graph.replay()
        torch.cuda.synchronize()
        check([m], [x], [y])


def test_no_tokens():
    m = Matrix(16, 64, 32, "f16", False, 3)
    slora.w4_matmul([m.handle], [0], 0, [0])
