"""GPU parity of the products of 8-bit integers against numpy in 64 bits: sums are exact, so that y is off by three roundings in fp32 (the sum's, two
products') and one to a 16-bit y."""
import numpy as np
import pytest
import torch

from dense_util import product, within
from paper_2311_03285_amd import slora

pytestmark = pytest.mark.gpu
DTYPES = {"f16": (slora.F16, torch.float16), "bf16": (slora.BF16, torch.bfloat16)}


class Matrix:
    def __init__(self, outputs, inputs, seed, dtype="f16", codes=None):
        rng = np.random.default_rng(seed)
        self.shape = outputs, inputs
        self.type = DTYPES[dtype][1]
        self.codes = rng.integers(-128, 128, (outputs, inputs), dtype=np.int8) if codes is None else codes
        self.scales = (rng.uniform(0.5, 1.5, outputs) / 70 / inputs ** 0.5).astype(np.float32)
        d_codes, d_scales = torch.from_numpy(self.codes).cuda(), torch.from_numpy(self.scales).cuda()
        self.packed = torch.full((slora.w8_bytes(outputs, inputs) + 16,), 0x5A, dtype=torch.uint8, device="cuda")
        self.handle = slora.w8_pack(outputs, inputs, DTYPES[dtype][0], d_codes.data_ptr(), d_scales.data_ptr(), self.packed.data_ptr())
        torch.cuda.synchronize()
        assert (self.packed[-16:] == 0x5A).all()


class X:
    """T rows of codes with anything behind them, and their scales"""

    def __init__(self, T, inputs, seed, pad=0, codes=None):
        rng = np.random.default_rng(seed)
        stride = -(-(inputs + pad) // 16) * 16
        all_codes = rng.integers(-128, 128, (T, stride), dtype=np.int8)
        if codes is not None:
            all_codes[:, :inputs] = codes
        self.codes, self.stride = all_codes[:, :inputs], stride
        self.scales = rng.uniform(0.5, 1.5, T).astype(np.float32) / 70
        self.d_codes, self.d_scales = torch.from_numpy(all_codes).cuda(), torch.from_numpy(self.scales).cuda()


def run(ms, xs, T, y16, y_pad=0, stream=None):
    ys = [torch.full((T + 1, m.shape[0] + y_pad), 7.0, dtype=m.type if y16 else torch.float32, device="cuda") for m in ms]
    torch.cuda.synchronize()
    (slora.w8_matmul_y16 if y16 else slora.w8_matmul)([m.handle for m in ms], [x.d_codes.data_ptr() for x in xs], [x.stride for x in xs],
                                                     [x.d_scales.data_ptr() for x in xs], T, [y.data_ptr() for y in ys], [y.stride(0) for y in ys], stream)
    torch.cuda.synchronize()
    for m, y in zip(ms, ys):
        assert (y[T] == 7.0).all() and (y[:, m.shape[0]:] == 7.0).all()
    return [y[:T, :m.shape[0]] for m, y in zip(ms, ys)]


def check(ms, xs, ys):
    for m, x, y in zip(ms, xs, ys):
        within(y, *product(x.codes[:len(y)], x.scales[:len(y)], m.codes, m.scales))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("y16", [False, True])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 513])
def test_tokens(T, y16, dtype):
    ms = [Matrix(200, 520, 1, dtype), Matrix(33, 520, 2, dtype)]
    x = X(T, 520, T)
    check(ms, [x, x], run(ms, [x, x], T, y16))


@pytest.mark.parametrize("outputs,inputs", [(1, 1), (15, 16), (16, 17), (17, 63), (33, 64), (100, 65), (129, 127), (128, 128), (200, 129), (300, 1000), (257, 4096),
                                            (130, 5003), (1000, 255), (31, 257)])
@pytest.mark.parametrize("T", [1, 20, 50, 70, 200, 300])
def test_shapes(outputs, inputs, T):
    m = Matrix(outputs, inputs, outputs + inputs, "bf16")
    for pad in (0, 48):
        x = X(T, inputs, T, pad)
        check([m], [x], run([m], [x], T, False, y_pad=pad))
    check([m], [x], run([m], [x], T, True, y_pad=3))


@pytest.mark.parametrize("outputs,T", [(3900, 3500), (4100, 3333), (8200, 1793)])
def test_many_tokens_and_outputs(outputs, T):
    m = Matrix(outputs, 200, 5)
    x = X(T, 200, 6)
    check([m], [x], run([m], [x], T, True))


# Shapes of tiles: of (outputs, tokens), the one whose rounds over 256 compute units cost least.  These sizes take each of the nine, with ends in both directions.
SHAPES = {(256, 256): (3900, 3500), (256, 192): (5100, 2000), (256, 128): (12250, 470), (128, 192): (15000, 333), (128, 128): (4090, 1000), (64, 128): (4090, 500),
          (64, 64): (4090, 200), (64, 32): (12280, 23), (32, 32): (4090, 63)}


@pytest.mark.parametrize("y16", [False, True])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_every_shape_of_tiles(shape, y16):
    outputs, T = SHAPES[shape]
    cost = {(256, 256): 1.7, (256, 192): 1.27, (256, 128): 0.95, (128, 192): 0.74, (128, 128): 0.56, (64, 128): 0.42, (64, 64): 0.3, (64, 32): 0.2, (32, 32): 0.18}
    took = min(cost, key=lambda s: -(-(-(-outputs // s[0]) * -(-T // s[1])) // 256) * cost[s])
    assert took == shape
    for more, pad in ((0, 0), (3, 0), (3, 6)):  # rows 16 bytes apart that end so or between, and rows that are not
        m = Matrix(outputs // 8 * 8 + more, 390, outputs)
        x = X(T, 390, 6, pad=16)
        check([m], [x], run([m], [x], T, y16, y_pad=-m.shape[0] % 8 + pad))


@pytest.mark.parametrize("shape", list(SHAPES))
def test_weights_too_large_for_the_caches(shape):
    """from 64 MiB of them on, other loads; a few tokens and the last ones are checked"""
    outputs, T = SHAPES[shape]
    inputs = -(-(68 << 20) // outputs)
    m, x = Matrix(outputs, inputs, 3), X(T, inputs, 4)
    y = run([m], [x], T, False)[0]
    rows = sorted({0, 1, T // 3, T // 2, T - 2, T - 1})
    within(y[rows], *product(x.codes[rows], x.scales[rows], m.codes, m.scales))


def test_graphs_on_two_streams_at_once():
    """nothing is shared between calls"""
    sets = [(Matrix(600 + 50 * i, 1500, i, "bf16"), X(T, 1500, i)) for i, T in enumerate((1, 40, 130, 500))]
    graphs, streams, ys = [], [], []
    for m, x in sets:
        T = len(x.codes)
        y, graph, stream = torch.zeros(T, m.shape[0], device="cuda"), torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            slora.w8_matmul([m.handle], [x.d_codes.data_ptr()], [x.stride], [x.d_scales.data_ptr()], T, [y.data_ptr()], [m.shape[0]], torch.cuda.current_stream())
        graphs.append(graph)
        streams.append(stream)
        ys.append(y)
    for _ in range(4):
        for y in ys:
            y.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (m, x), y in zip(sets, ys):
            check([m], [x], [y])


@pytest.mark.parametrize("T", [1, 40, 70, 300])
def test_matrices_of_different_shapes(T):
    shapes = [(16, 64), (100, 8), (3, 2048), (512, 512), (31, 136), (64, 64), (1, 1000), (40, 3200)]
    ms = [Matrix(o, i, o, "bf16") for o, i in shapes]
    xs = [X(T, i, o, pad=o % 3 * 16) for o, i in shapes]
    check(ms, xs, run(ms, xs, T, False, stream=torch.cuda.Stream()))
    check(ms, xs, run(ms, xs, T, True, y_pad=5))


@pytest.mark.parametrize("T", [1, 30, 60, 70])
def test_the_largest_sums_are_exact(T):
    """-128 * -128 at the most inputs is 2^31 - 2^14; -128 * 127 of them is the other end"""
    n = 131071
    for x_code in (-128, 127):
        m = Matrix(20, n, 1, codes=np.full((20, n), -128, np.int8))
        x = X(T, n, 1, codes=np.full((T, n), x_code, np.int8))
        x.d_scales.fill_(1.0)
        y = run([m], [x], T, False)[0].double().cpu().numpy()
        want = np.float32(-128 * x_code * n).astype(np.float64) * m.scales  # one rounding of the sum, one of the product
        assert (np.abs(y - want) <= 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("T", [9, 64, 256])
def test_every_code_times_every_place(T):
    """one input at a time: each weight by itself"""
    m = Matrix(64, 256, 5)
    m2 = Matrix(64, 256, 5)
    eye = np.zeros((256, 256), np.int8)
    np.fill_diagonal(eye, 1)
    for t0 in range(0, 256, T):
        codes = eye[t0:t0 + T]
        x = X(len(codes), 256, 1, codes=codes)
        x.d_scales.fill_(1.0)
        y = run([m, m2], [x, x], len(codes), False)
        want = m.codes.T[t0:t0 + T].astype(np.float32) * m.scales
        assert np.array_equal(y[0].cpu().numpy(), want) and torch.equal(y[0], y[1])


@pytest.mark.parametrize("T", [5, 40, 100, 300])
def test_a_spoiled_token_leaves_the_others_alone(T):
    m = Matrix(150, 300, 4)
    x = X(T, 300, 3)
    clean = run([m], [x], T, False)[0].clone()
    x.d_scales[3], x.d_scales[T - 1] = float("nan"), float("inf")
    y = run([m], [x], T, False)[0]
    others = [t for t in range(T) if t not in (3, T - 1)]
    assert torch.equal(y[others], clean[others]) and torch.isnan(y[3]).all() and not torch.isfinite(y[T - 1]).any()


def test_scales_far_apart():
    """the sum times one scale, then the other: no product of scales that leaves fp32's range"""
    m = Matrix(40, 500, 4)
    for by_x, by_w in ((2.0 ** -100, 2.0 ** 60), (2.0 ** 90, 2.0 ** -110)):
        m.packed.view(torch.float32)[m.packed.numel() // 4 - 4 - 48:-4].mul_(by_w)
        torch.cuda.synchronize()
        for T in (3, 90):
            x = X(T, 500, 1)
            x.scales = x.scales * np.float32(by_x)
            x.d_scales.mul_(by_x)
            ref, bound = product(x.codes, x.scales, m.codes, m.scales.astype(np.float64) * by_w)
            within(run([m], [x], T, False)[0], ref, bound)
        m.packed.view(torch.float32)[m.packed.numel() // 4 - 4 - 48:-4].mul_(1 / by_w)
        torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 50, 130])
def test_a_graph_replays_the_product(T):
    m = Matrix(300, 700, 3, "bf16")
    x, y = X(T, 700, 1), torch.zeros(T, 300, device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        slora.w8_matmul([m.handle], [x.d_codes.data_ptr()], [x.stride], [x.d_scales.data_ptr()], T, [y.data_ptr()], [300], torch.cuda.current_stream())
    for seed in range(3):
        new = X(T, 700, 10 + seed)
        x.d_codes.copy_(new.d_codes)
        x.d_scales.copy_(new.d_scales)
        y.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        check([m], [new], [y])


@pytest.mark.parametrize("T", [1, 64, 200])
def test_calls_repeat_to_the_bit(T):
    ms = [Matrix(1000, 2000, 3), Matrix(520, 2000, 4)]
    x = X(T, 2000, 1)
    first = [y.clone() for y in run(ms, [x, x], T, True)]
    for _ in range(3):
        for a, b in zip(first, run(ms, [x, x], T, True)):
            assert torch.equal(a, b)


def test_tokens_do_not_change_with_the_batch():
    m = Matrix(700, 900, 3)
    x = X(600, 900, 1)
    whole = run([m], [x], 600, True)[0]
    for T in (1, 16, 40, 70, 128, 300):
        assert torch.equal(run([m], [x], T, True)[0], whole[:T])


def test_rows_far_apart_and_outputs_behind_4_GiB():
    T, O = 70000, 32771
    m = Matrix(O, 40, 3)
    x = X(T, 40, 1)
    y = torch.empty((T, O), dtype=torch.float16, device="cuda")
    slora.w8_matmul_y16([m.handle], [x.d_codes.data_ptr()], [x.stride], [x.d_scales.data_ptr()], T, [y.data_ptr()], [O])
    torch.cuda.synchronize()
    rows = [0, 1, 255, 256, 40000, 65535, 65536, 69887, 69888, T - 1]
    within(y[rows], *product(x.codes[rows], x.scales[rows], m.codes, m.scales))
    # rows of x 2^22 bytes apart: 300 of them pass 2^30
    x = torch.zeros((300, 1 << 22), dtype=torch.int8, device="cuda")
    small = X(300, 40, 2)
    x[:, :40] = torch.from_numpy(small.codes).cuda()
    y = torch.empty((300, O), dtype=torch.float16, device="cuda")
    slora.w8_matmul_y16([m.handle], [x.data_ptr()], [1 << 22], [small.d_scales.data_ptr()], 300, [y.data_ptr()], [O])
    torch.cuda.synchronize()
    within(y, *product(small.codes, small.scales, m.codes, m.scales))


def test_no_tokens():
    m = Matrix(16, 64, 3)
    slora.w8_matmul([m.handle], [0], [0], [0], 0, [0], [0])


def test_refusals():
    m, other = Matrix(16, 64, 3), Matrix(16, 64, 3, "bf16")
    x, y = X(4, 64, 1), torch.zeros(2, 8, 16, device="cuda")
    good = dict(handles=[m.handle], xs=[x.d_codes.data_ptr()], x_strides=[64], x_scales=[x.d_scales.data_ptr()], T=4, ys=[y.data_ptr()], y_strides=[16])

    def refused(text, **kw):
        with pytest.raises(slora.SloraError, match=text) as e:
            slora.w8_matmul(**{**good, **kw})
        assert e.value.code == slora.EINVAL

    refused("negative", T=-1)
    refused("is NULL", xs=[0])
    refused("is NULL", x_scales=[0])
    refused("is NULL", ys=[0])
    refused("16-byte", xs=[x.d_codes.data_ptr() + 8])
    refused("16-byte", ys=[y.data_ptr() + 4])
    refused("4-byte", x_scales=[x.d_scales.data_ptr() + 2])
    for stride in (0, 48, 72, -64, (1 << 22) + 16):
        refused("x_stride", x_strides=[stride])
    for stride in (15, -16, 1 << 30):
        refused("y_stride", y_strides=[stride])
    refused("another type", **{k: v * 2 for k, v in good.items() if k != "T"} | {"handles": [m.handle, other.handle]})
    refused("same buffer", **{k: v * 2 for k, v in good.items() if k != "T"})
    refused("in \\[1, 8\\]", **{k: v * 9 for k, v in good.items() if k != "T"})
    with pytest.raises(ValueError):
        slora.w8_matmul(**{**good, "x_strides": [64, 64]})
    torch.cuda.synchronize()
    assert (y == 0).all()
