"""GPU parity of the norms around a block and of rows in 8 bits against numpy in 64 bits, with the bounds of dense_util."""
import numpy as np
import pytest
import torch

import dense_util as du
from paper_2311_03285_amd import slora

pytestmark = pytest.mark.gpu
DTYPES = {"f16": (slora.F16, torch.float16), "bf16": (slora.BF16, torch.bfloat16)}
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 511, 512, 513, 519, 520, 1000, 1023, 1024, 1025, 1032, 2048, 4096, 5003, 8192, 10247, 16384, 16391, 16392, 16400, 20001, 32767, 32768]


def rows(T, width, dtype, seed, pad=0, size=1.0):
    """T rows with a value behind each that nothing may touch"""
    rng = np.random.default_rng(seed)
    stride = -(-(width + pad) // 8) * 8
    a = torch.full((T, stride), 5.0, dtype=dtype)
    a[:, :width] = torch.from_numpy(rng.standard_normal((T, width)) * size).to(dtype)
    return a.cuda()


def vector(width, dtype, seed, mean):
    return torch.from_numpy(mean + 0.3 * np.random.default_rng(seed).standard_normal(width)).to(dtype).cuda()


def np64(a, width=None):
    return None if a is None else (a if width is None else a[..., :width]).double().cpu().numpy()


class Norm:
    def __init__(self, width, dtype, layer=False, post=False, bias=False, h32=False, weights=True, eps=1e-5, scale=1.0, seed=0):
        self.width, self.layer, self.post, self.eps, self.scale, self.h32 = width, layer, post, np.float64(np.float32(eps)), np.float64(np.float32(scale)), h32
        lib, self.type = DTYPES[dtype]
        t = self.type
        self.pre = (vector(width, t, seed + 1, 1.0) if weights else None, vector(width, t, seed + 2, 0.0) if bias else None)
        self.posts = (vector(width, t, seed + 3, 1.0) if weights and post else None, vector(width, t, seed + 4, 0.0) if bias and post else None)
        flags = slora.NORM_LAYER * layer | slora.NORM_POST * post | slora.NORM_H32 * h32
        at = [None if v is None else v.data_ptr() for v in (*self.posts, *self.pre)]
        self.handle = slora.norm_init(width, lib, flags, eps, scale, *at)

    def __call__(self, h, block=None, gate=None, h_out=True, x=True, codes=True, stream=None):
        T, n = h.shape[0], self.width
        out = {}
        kw = {}
        if block is not None:
            kw.update(block=block.data_ptr(), block_stride=block.stride(0))
        if gate is not None:
            kw.update(gate=gate.data_ptr(), gate_stride=0 if gate.dim() == 1 else gate.stride(0))
        if h_out is not False:
            out["h"] = torch.full((T + 1, h.shape[1]), 9.0, dtype=h.dtype, device="cuda") if h_out is True else h_out
            kw.update(h_out=out["h"].data_ptr(), h_out_stride=out["h"].stride(0))
        if x is not False:
            out["x"] = torch.full((T + 1, -(-n // 8) * 8 + 8), 9.0, dtype=self.type, device="cuda") if x is True else x
            kw.update(x=out["x"].data_ptr(), x_stride=out["x"].stride(0))
        if codes:
            out["codes"] = torch.full((T + 1, -(-n // 16) * 16 + 16), 99, dtype=torch.int8, device="cuda")
            out["scales"] = torch.full((T + 1,), 9.0, device="cuda")
            kw.update(codes=out["codes"].data_ptr(), codes_stride=out["codes"].stride(0), scales=out["scales"].data_ptr())
        torch.cuda.synchronize()
        slora.norm_apply(self.handle, T, h.data_ptr(), h.stride(0), **kw, stream=stream)
        torch.cuda.synchronize()
        for name, a in out.items():  # nothing behind the rows is touched
            mark = 99 if name == "codes" else 9.0
            if (name == "h" and h_out is True) or (name == "x" and x is True) or name in ("codes", "scales"):
                assert (a[T] == mark).all(), name
                if name != "scales":
                    assert (a[:, n:] == mark).all(), name
                out[name] = a[:T] if name == "scales" else a[:T, :n]
            else:
                out[name] = a[:T, :n]
        return out

    def reference(self, h, block=None, gate=None):
        n = self.width
        post = tuple(np64(v) for v in self.posts) if self.post and block is not None else None
        return du.norm(np64(h, n), np64(block, n), np64(gate, n), self.scale, post, tuple(np64(v) for v in self.pre), self.layer, self.eps)

    def check(self, h, block=None, gate=None, **kw):
        ref_h, eh, ref_x, ex = self.reference(h, block, gate)
        out = self(h, block, gate, **kw)
        if "h" in out:
            du.within(out["h"], ref_h, eh)
        if "x" in out:
            du.within(out["x"], ref_x, ex)
        if "codes" in out:
            du.codes_within(out["codes"], out["scales"], ref_x, ex)
        return out


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, dtype):
    t = DTYPES[dtype][1]
    for k, (layer, post, bias, h32) in enumerate([(False, False, False, False), (False, True, False, False), (True, True, True, True), (True, False, True, False),
                                                  (False, True, True, True)]):
        m = Norm(width, dtype, layer, post, bias, h32, scale=0.7, seed=width)
        h = rows(3, width, torch.float32 if h32 else t, k, size=3.0)
        m.check(h, rows(3, width, t, k + 10, pad=8 * k), vector(width, t, k, 0.5) if k % 2 else rows(3, width, t, 77, pad=16))


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 300])
@pytest.mark.parametrize("width", [8, 130, 520, 1100, 4096])
def test_tokens(T, width):
    m = Norm(width, "f16", post=True, seed=3)
    h, block = rows(T, width, torch.float16, 1), rows(T, width, torch.float16, 2)
    whole = m.check(h, block)
    one = m(h[T - 1:], block[T - 1:])
    for name in whole:
        assert torch.equal(one[name][0], whole[name][T - 1]), name  # whatever else is in the batch


@pytest.mark.parametrize("width", [96, 1024, 5003, 20000])
def test_any_subset_of_outputs(width):
    t = torch.bfloat16
    m = Norm(width, "bf16", layer=True, bias=True)
    h, block, gate = rows(4, width, t, 1), rows(4, width, t, 2), vector(width, t, 3, 0.3)
    full = m.check(h, block, gate)
    for keep in ({"h_out"}, {"x"}, {"codes"}, {"h_out", "codes"}, {"x", "codes"}):
        out = m(h, block, gate, **{k: k in keep for k in ("h_out", "x", "codes")})
        for name, a in out.items():
            assert torch.equal(a, full[name])
    m.check(h)  # a norm alone: h_out is h
    assert torch.equal(m(h)["h"], h[:, :width])


def test_without_weights_and_with_an_eps_that_matters():
    for layer in (False, True):
        m = Norm(777, "f16", layer=layer, post=True, weights=False, eps=0.5)
        m.check(rows(5, 777, torch.float16, 1), rows(5, 777, torch.float16, 2))


def test_in_place():
    t = torch.float16
    for width in (40, 1001, 8192):
        m = Norm(width, "f16", post=True, seed=1)
        h, block = rows(6, width, t, 1), rows(6, width, t, 2)
        want = m(h, block)
        h2, b2 = h.clone(), block.clone()
        got = m(h2, b2, h_out=h2, x=b2)
        for name in want:
            assert torch.equal(got[name], want[name]), name
        assert (h2[:, width:] == 5.0).all() and (b2[:, width:] == 5.0).all()


@pytest.mark.parametrize("width", [64, 700, 4096, 17000])
@pytest.mark.parametrize("layer", [False, True])
def test_magnitudes_whose_squares_leave_the_range(width, layer):
    """bfloat16 rows of 2^-110 .. 2^120, without eps: every row by itself"""
    m = Norm(width, "bf16", layer=layer, eps=0.0)
    h = rows(9, width, torch.bfloat16, 1)
    for t, e in enumerate([-110, -90, -70, -30, 0, 40, 60, 90, 120]):
        h[t, :width] = h[t, :width] * 2.0 ** e
    m.check(h)
    m32 = Norm(width, "bf16", layer=layer, eps=0.0, h32=True)
    m32.check(h.float())


def test_a_mean_far_from_the_spread():
    """differences are taken of the values, not of sums of squares"""
    m = Norm(4096, "f16", layer=True, h32=True)
    h = rows(4, 4096, torch.float32, 1) + torch.tensor([0.0, 100.0, -3000.0, 20000.0], device="cuda")[:, None]
    m.check(h)


@pytest.mark.parametrize("width", [33, 4096])
def test_infinities_and_nans_stay_in_their_rows(width):
    t = torch.bfloat16
    m = Norm(width, "bf16", post=True)
    h, block = rows(6, width, t, 1), rows(6, width, t, 2)
    clean = m(h, block)
    h[1, 5], block[3, 7], h[4, 0] = float("inf"), float("nan"), float("-inf")
    out = m(h, block)
    for row in (0, 2, 5):
        for name in out:
            assert torch.equal(out[name][row], clean[name][row])
    assert torch.isnan(out["x"][1, 5]) and (out["x"][1, 6:] == 0).all()     # inf / inf, finite / inf
    assert torch.isnan(out["x"][3]).all() and torch.isnan(out["h"][3]).all()
    for row in (1, 3, 4):
        assert torch.isnan(out["scales"][row]) and (out["codes"][row] == 0).all()
    assert out["h"][1, 5] == float("inf") and out["h"][4, 0] == float("-inf")


def test_rows_of_zeros():
    for layer in (False, True):
        out = Norm(600, "f16", layer=layer)(torch.zeros(3, 600, dtype=torch.float16, device="cuda"))
        assert (out["x"] == 0).all() and (out["codes"] == 0).all() and (out["scales"] == np.float32(2.0 ** -100) / np.float32(127)).all()
        out = Norm(600, "f16", layer=layer, eps=0.0)(torch.zeros(3, 600, dtype=torch.float16, device="cuda"))
        assert torch.isnan(out["x"]).all() and torch.isnan(out["scales"]).all()  # 0 / 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("width", WIDTHS + [40000, 65535, 65536])
def test_quantize_is_the_definition(width, dtype):
    lib, t = DTYPES[dtype]
    T = 5
    x = rows(T, width, t, width, pad=width % 5)
    x[1, :width] *= 1e-4
    x[2, :width] = 0.0
    x[3, width // 2] = 300.0
    codes, scales = torch.full((T + 1, -(-width // 16) * 16 + 16), 99, dtype=torch.int8, device="cuda"), torch.full((T + 1,), 9.0, device="cuda")
    y = torch.full((T + 1, x.shape[1]), 9.0, dtype=t, device="cuda")
    slora.w8_quantize(T, width, lib, slora.ACT_NONE, x.data_ptr(), x.stride(0), y=y.data_ptr(), y_stride=y.stride(0), codes=codes.data_ptr(),
                      codes_stride=codes.stride(0), scales=scales.data_ptr())
    torch.cuda.synchronize()
    want, by = du.codes_of(x[:, :width].float().cpu().numpy())
    assert np.array_equal(codes[:T, :width].cpu().numpy(), want) and np.array_equal(scales[:T].cpu().numpy(), by)
    assert torch.equal(y[:T, :width], x[:, :width]) and (y[T] == 9.0).all() and (y[:, width:] == 9.0).all()
    assert (codes[T] == 99).all() and (codes[:, width:] == 99).all() and scales[T] == 9.0


@pytest.mark.parametrize("width", [24, 1000])
def test_quantize_ties_and_extremes(width):
    """halves go to the even code; subnormal rows count as 2^-100; infinities and NaN spoil their row alone"""
    x = torch.zeros((6, width), dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[0, 1:7] = 127.0, torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, -2.5], device="cuda").bfloat16()
    x[1, 3] = 2.0 ** -120
    x[2, 3], x[2, 4] = float("inf"), 1.0
    x[3, 3], x[3, 4] = float("nan"), 1.0
    x[4, 0], x[4, 1] = 3.0e38, -3.0e38
    x[5, :] = -1.0
    codes, scales = torch.empty((6, -(-width // 16) * 16), dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    slora.w8_quantize(6, width, slora.BF16, slora.ACT_NONE, x.data_ptr(), width, codes=codes.data_ptr(), codes_stride=codes.stride(0), scales=scales.data_ptr())
    torch.cuda.synchronize()
    c = codes[:, :width].cpu().numpy()
    assert c[0, :7].tolist() == [127, 0, 2, 2, 0, -2, -2]
    assert (c[1] == 0).all() and scales[1] == np.float32(2.0 ** -100) / np.float32(127)
    assert (c[2:4] == 0).all() and torch.isnan(scales[2:4]).all()
    assert c[4, :2].tolist() == [127, -127] and (c[5] == -127).all()
    want, by = du.codes_of(x.float().cpu().numpy())
    assert np.array_equal(c, want) and np.array_equal(scales.cpu().numpy(), by, equal_nan=True)


def act(kind, g):
    with np.errstate(over="ignore"):
        u = g if kind == slora.ACT_SILU else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
        return g / (1 + np.exp(-u)), np.abs(u)


@pytest.mark.parametrize("kind", [slora.ACT_SILU, slora.ACT_GELU])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("width", [1, 9, 64, 1000, 4096, 13007, 40000])
def test_gated(width, dtype, kind):
    """exp(-u) is off by two roundings of u's (|u| E each), u by five, and by its own two steps; then a sum, a quotient and a product"""
    lib, t = DTYPES[dtype]
    T = 4
    x, gate = rows(T, width, t, 1, pad=8), rows(T, width, t, 2, size=3.0)
    gate[1, :width] *= 5
    y, codes, scales = torch.empty_like(x), torch.empty((T, -(-width // 16) * 16), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    slora.w8_quantize(T, width, lib, kind, x.data_ptr(), x.stride(0), gate.data_ptr(), gate.stride(0), y.data_ptr(), y.stride(0), codes.data_ptr(), codes.stride(0),
                      scales.data_ptr())
    torch.cuda.synchronize()
    f, u = act(kind, np64(gate, width))
    ref = f * np64(x, width)
    bound = du.E * np.abs(ref) * (7 * u + 2 + 4)
    # (where exp(-u) passes fp32's range, u < -88, the result is 0 and the value below 2^-120 of the gate)
    bound = bound + np.abs(np64(gate, width) * np64(x, width)) * 2.0 ** -120
    du.within(y[:, :width], ref, bound)
    du.codes_within(codes[:, :width], scales, ref, bound)
    again = x.clone()
    slora.w8_quantize(T, width, lib, kind, again.data_ptr(), x.stride(0), gate.data_ptr(), gate.stride(0), again.data_ptr(), x.stride(0))
    torch.cuda.synchronize()
    assert torch.equal(again[:, :width], y[:, :width]) and (again[:, width:] == 5.0).all()


def test_gates_at_the_ends():
    x = torch.ones((1, 16), dtype=torch.bfloat16, device="cuda")
    gate = torch.zeros((1, 16), dtype=torch.bfloat16, device="cuda")
    gate[0, :8] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1e30, -1e30, 100.0, -100.0, -0.0], device="cuda").bfloat16()
    for kind in (slora.ACT_SILU, slora.ACT_GELU):
        y = torch.empty_like(x)
        slora.w8_quantize(1, 16, slora.BF16, kind, x.data_ptr(), 16, gate.data_ptr(), 16, y.data_ptr(), 16)
        torch.cuda.synchronize()
        v = y[0].float().cpu().numpy()
        assert v[0] == np.inf and np.isnan(v[1]) and np.isnan(v[2]) and v[3] == gate[0, 3].item() and abs(v[4]) == 0 and v[5] == 100 and abs(v[6]) < 1e-38 and v[7] == 0


@pytest.mark.parametrize("width", [200, 4096])
def test_graphs_and_streams(width):
    t = torch.float16
    m = Norm(width, "f16", post=True)
    h, block = rows(9, width, t, 1), rows(9, width, t, 2)
    x, h2 = torch.empty_like(h), torch.empty_like(h)
    codes, scales = torch.empty((9, -(-width // 16) * 16), dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    y = torch.empty_like(h)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        s = torch.cuda.current_stream()
        slora.norm_apply(m.handle, 9, h.data_ptr(), h.stride(0), block.data_ptr(), block.stride(0), h_out=h2.data_ptr(), h_out_stride=h2.stride(0), x=x.data_ptr(),
                         x_stride=x.stride(0), stream=s)
        slora.w8_quantize(9, width, slora.F16, slora.ACT_SILU, x.data_ptr(), x.stride(0), h2.data_ptr(), h2.stride(0), y.data_ptr(), y.stride(0), codes.data_ptr(),
                          codes.stride(0), scales.data_ptr(), stream=s)
    for seed in range(4):
        h.copy_(rows(9, width, t, 20 + seed))
        block.copy_(rows(9, width, t, 30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        want = m(h, block, codes=False, stream=torch.cuda.Stream())
        assert torch.equal(want["x"], x[:, :width]) and torch.equal(want["h"], h2[:, :width])
        c, s2, y2 = torch.empty_like(codes), torch.empty_like(scales), torch.empty_like(y)
        slora.w8_quantize(9, width, slora.F16, slora.ACT_SILU, x.data_ptr(), x.stride(0), h2.data_ptr(), h2.stride(0), y2.data_ptr(), y2.stride(0), c.data_ptr(),
                          c.stride(0), s2.data_ptr())
        torch.cuda.synchronize()
        assert torch.equal(c[:, :width], codes[:, :width]) and torch.equal(s2, scales) and torch.equal(y2[:, :width], y[:, :width])


def test_rows_behind_4_GiB_and_more_rows_than_a_grid_is_wide():
    T, width = (1 << 20) + 5, 2056  # a workgroup a row
    h = torch.empty((T, width), dtype=torch.float16, device="cuda")
    h.normal_()
    m = Norm(width, "f16")
    x = torch.empty_like(h)
    slora.norm_apply(m.handle, T, h.data_ptr(), width, x=x.data_ptr(), x_stride=width)
    torch.cuda.synchronize()
    for t in (0, 1 << 19, (1 << 20) - 1, 1 << 20, T - 1):
        one = m(h[t:t + 1], h_out=False, codes=False)
        assert torch.equal(one["x"][0], x[t])
    codes, scales = torch.empty((T, 2064), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    slora.w8_quantize(T, width, slora.F16, slora.ACT_NONE, h.data_ptr(), width, codes=codes.data_ptr(), codes_stride=2064, scales=scales.data_ptr())
    torch.cuda.synchronize()
    for t in (0, (1 << 20) - 1, 1 << 20, T - 1):
        want, by = du.codes_of(h[t:t + 1].float().cpu().numpy())
        assert np.array_equal(codes[t:t + 1, :width].cpu().numpy(), want) and scales[t].item() == by[0]


@pytest.mark.parametrize("width", [100, 515, 1000, 1003, 4096, 5003, 20000, 20005])
def test_rows_too_large_for_the_caches(width):
    """from 64 MiB of them on, other loads: every row as in a call of few"""
    T, t = (70 << 20) // (4 * width) + 1, torch.bfloat16
    some = [0, 1, T // 2, T - 1]
    for h32 in (False, True):
        m = Norm(width, "bf16", layer=h32, post=True, bias=True, h32=h32)
        h, block = rows(T, width, torch.float32 if h32 else t, 1), rows(T, width, t, 2)
        whole, few = m(h, block), m(h[some].contiguous(), block[some].contiguous())
        for name in few:
            assert torch.equal(whole[name][some], few[name]), name
    for gate in (None, block):
        kw = {} if gate is None else dict(gate=gate.data_ptr(), gate_stride=gate.stride(0))
        x, kind = (block, slora.ACT_NONE) if gate is None else (whole["x"].contiguous() if width % 8 == 0 else block, slora.ACT_SILU)
        x = torch.cat([x, x]) if gate is None else x
        n, out = x.shape[0], {}
        for which in ("whole", "few"):
            pick = list(range(n)) if which == "whole" else some
            a = x if which == "whole" else x[some].contiguous()
            g = gate if which == "whole" or gate is None else gate[some].contiguous()
            if g is not None:
                kw = dict(gate=g.data_ptr(), gate_stride=g.stride(0))
            codes, scales = torch.empty((len(pick), -(-width // 16) * 16), dtype=torch.int8, device="cuda"), torch.empty(len(pick), device="cuda")
            slora.w8_quantize(len(pick), width, slora.BF16, kind, a.data_ptr(), a.stride(0), codes=codes.data_ptr(), codes_stride=codes.stride(0), scales=scales.data_ptr(), **kw)
            torch.cuda.synchronize()
            out[which] = codes[:, :width], scales
        assert torch.equal(out["whole"][0][some], out["few"][0]) and torch.equal(out["whole"][1][some], out["few"][1])


def test_no_tokens():
    m = Norm(64, "f16")
    slora.norm_apply(m.handle, 0, 0, 0)
    slora.w8_quantize(0, 64, slora.F16, slora.ACT_NONE, 0, 0)
