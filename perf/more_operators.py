"""The dense side of a served layer in 8-bit integers: what runs between its products, and the products of prompts.

Three operators that a serving loop calls around LoRA and attention:

  norm      the junction of two blocks: the last block's output, normalised and gated if the model does so, is added onto the
            residual stream, which is normalised for the next block, in 16 bits, in 8-bit codes with a scale per token, or both
  quantize  rows to 8-bit codes with a scale per token, of x or of act(gate) * x; or that product alone, in 16 bits
  w8        products of 8-bit codes of x and of weights with a scale for each token and for each output

A case of kind "norm", "quantize" or "w8" is one call; one of kind "qkv" or "mlp" is a run of them as a layer makes it: norm and
the projections that read it, or norm, the two wide projections, their gated product in 8 bits, and the one back.

A row of codes is that of v with a = max(|v|, 2^-100): scale = a / 127, code = v * (127 / a) rounded to nearest, ties to even, where
quotient and product are fp32.
"""
from __future__ import annotations

import torch

own = False

_DEVICE = "cuda"
_LEAST = 2.0 ** -100
_EPS = 1e-5


def listed():
    norm = {"op": "norm", "tokens": 1, "width": 4096, "kind": "rms", "post": False, "gate": "none", "bias": False, "h": "16", "pad": 0, "scale": 1.0, "dtype": "f16"}
    quantize = {"op": "quantize", "tokens": 1, "width": 4096, "act": "none", "pad": 0, "dtype": "f16"}
    w8 = {"op": "w8", "tokens": 1, "inputs": 4096, "outputs": 4096, "n": 1, "pad": 0, "y": "16", "dtype": "f16"}
    qkv = {"op": "qkv", "tokens": 1, "width": 4096, "outputs": 4096, "kind": "rms", "post": False, "dtype": "f16"}
    mlp = {"op": "mlp", "tokens": 1, "width": 4096, "wide": 16384, "act": "silu", "kind": "rms", "post": False, "dtype": "f16"}

    def case(base, name, **kw):
        return {"name": name, **base, **kw}

    return [
        # a single interactive user's token between two blocks: latency
        case(norm, "norm_1"),
        # a prefill batch of a wide model that normalises a block's output too and scales it by channel
        case(norm, "norm_prompt", tokens=8192, width=8192, post=True, gate="channel", scale=0.7, dtype="bf16"),
        # uneven sizes: layer norms with biases, an odd width, rows apart, a residual stream in fp32, a gate for every token
        case(norm, "norm_ragged", tokens=777, width=5003, kind="layer", post=True, gate="token", bias=True, h="32", pad=24),
        # a single token's attention output before its projection
        case(quantize, "quantize_1"),
        # the same of a prefill batch
        case(quantize, "quantize_prompt", tokens=4096, width=5120, dtype="bf16"),
        # the gated product of a prefill batch in 16 bits, before a product that is not in 8; an odd width, rows apart
        case(quantize, "gated_ragged", tokens=3001, width=13007, act="silu", pad=41),
        # the four attention projections of a single token
        case(w8, "product_1", n=4),
        # a decode batch through the wide matrices of a layer
        case(w8, "product_32", tokens=32, inputs=5120, outputs=20480, n=2, dtype="bf16"),
        # uneven sizes: tokens, inputs and outputs that no tile divides, rows apart, outputs in fp32
        case(w8, "product_ragged", tokens=333, inputs=3083, outputs=5003, n=3, pad=32, y="32"),
        # a prefill batch of a wide model
        case(w8, "product_prompt", tokens=8192, inputs=8192, outputs=8192, dtype="bf16"),
        # iteration-level batching on a small node: 24 requests' tokens through the first half of an attention block
        case(qkv, "qkv_decode", tokens=24),
        # a chunk of prompts through the whole feed-forward block
        case(mlp, "mlp_prompt", tokens=2048, width=5120, wide=20480, post=True, dtype="bf16"),
    ]


def draw(rng):
    """One more case of the kinds and ranges above."""

    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    most = [work(c) for c in listed()]
    top = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["norm", "norm", "quantize", "w8", "w8", "w8", "qkv", "mlp"])
        c = {"op": op, "tokens": spread(1, 16384), "dtype": rng.choice(["f16", "bf16"])}
        width = rng.choice([64, 128, 1024, 2048, 4096, 5120, 8192, 16384, spread(16, 16384), spread(16, 16384)])
        if op in ("norm", "qkv", "mlp"):
            c.update(width=width, kind=rng.choice(["rms", "rms", "layer"]), post=rng.random() < 0.5)
        if op == "norm":
            c.update(gate=rng.choice(["none", "channel", "token"]), bias=rng.random() < 0.3, h=rng.choice(["16", "16", "32"]), pad=rng.choice([0, 0, spread(1, 512)]),
                     scale=rng.choice([1.0, 1.0, 0.25 + rng.random()]))
        elif op == "quantize":
            c.update(width=rng.choice([width, spread(16, 32768)]), act=rng.choice(["none", "none", "silu", "gelu"]), pad=rng.choice([0, 0, spread(1, 512)]))
        elif op == "w8":
            c.update(inputs=rng.choice([width, spread(16, 20480)]), outputs=rng.choice([1024, 4096, 5120, 8192, spread(1, 20480)]), n=rng.choice([1, 1, 2, 3, 4, 8]),
                     pad=rng.choice([0, 0, spread(16, 512)]), y=rng.choice(["16", "16", "32"]))
        elif op == "qkv":
            c.update(outputs=width)
        else:
            c.update(wide=rng.choice([4 * width, spread(16, 20480)]), act=rng.choice(["silu", "gelu"]))
        w = work(c)
        if w["bytes"] <= top["bytes"] and w["flops"] <= top["flops"]:
            return c


# ---- what a case means ---------------------------------------------------------------------------
def work(case):
    """norm: the residual stream and the block's output read, both results written; quantize: what is read, codes or products; w8: codes,
    scales and y; a run of them: what goes in and comes out, and the weights."""
    T, op = case["tokens"], case["op"]
    if op == "norm":
        n = case["width"]
        per_token = n * (2 * (4 if case["h"] == "32" else 2) + 2 + 2 + (2 if case["gate"] == "token" else 0))
        vectors = 1 + (1 if case["post"] else 0) + (1 if case["gate"] == "channel" else 0)
        return {"bytes": T * per_token + 2 * n * vectors, "flops": 8 * T * n}
    if op == "quantize":
        n = case["width"]
        return {"bytes": T * n * (2 + 1) + 4 * T if case["act"] == "none" else T * n * (4 + 2), "flops": (2 if case["act"] == "none" else 6) * T * n}
    if op == "w8":
        I, O, n = case["inputs"], case["outputs"], case["n"]
        return {"bytes": n * (O * I + 4 * O + T * O * (4 if case["y"] == "32" else 2)) + T * (I + 4), "flops": 2 * n * T * O * I}
    n = case["width"]
    if op == "qkv":
        O = case["outputs"]
        return {"bytes": T * n * 8 + 3 * (O * (n + 4) + 2 * T * O), "flops": 6 * T * O * n}
    wide = case["wide"]
    return {"bytes": T * n * 8 + 3 * n * wide + 8 * wide + 4 * n, "flops": 6 * T * n * wide}


def _type(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _up(n, to):
    return -(-n // to) * to


# ---- inputs ----------------------------------------------------------------------------------------
class _State:
    def __init__(self, case):
        self.case = case
        self.close = []

    def __del__(self):
        for end, handle in self.close:
            end(handle)


def _rows(T, n, pad, dtype, gen, size=1.0):
    """T rows of n values, each in a place of n + pad of its own"""
    return (torch.randn((T, _up(n + pad, 8)), device=_DEVICE, generator=gen) * size).to(dtype)


def _vector(n, dtype, gen, mean, size):
    return (mean + size * torch.randn((n,), device=_DEVICE, generator=gen)).to(dtype)


def _weights(s, O, I, gen):
    """codes of normal weights, a scale per output: y of the size of x"""
    codes = (torch.randn((O, I), device=_DEVICE, generator=gen) * 35).round_().clamp_(-127, 127).to(torch.int8)
    s.weights.append((codes, (0.5 + torch.rand((O,), device=_DEVICE, generator=gen)) / (35 * I ** 0.5)))


def _norm_inputs(s, T, n, gen, post, gate="none", bias=False, h32=False, pad=0):
    t = _type(s.case)
    s.h = _rows(T, n, pad, torch.float32 if h32 else t, gen, 3.0)
    s.h[:, :n:97] *= 8  # a few channels stand out, as they do in residual streams
    s.block = _rows(T, n, pad, t, gen)
    s.gate = None if gate == "none" else _vector(n, t, gen, 0.5, 0.3) if gate == "channel" else _rows(T, n, pad, t, gen)
    s.post_w, s.post_b = (_vector(n, t, gen, 1.0, 0.2), _vector(n, t, gen, 0.0, 0.2) if bias else None) if post else (None, None)
    s.pre_w, s.pre_b = _vector(n, t, gen, 1.0, 0.2), _vector(n, t, gen, 0.0, 0.2) if bias else None
    s.h_out, s.x = torch.empty_like(s.h), torch.empty_like(s.block)


def _inputs(case, seed):
    s = _State(case)
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(seed)
    T, t, op = case["tokens"], _type(case), case["op"]
    s.weights = []
    if op == "norm":
        _norm_inputs(s, T, case["width"], gen, case["post"], case["gate"], case["bias"], case["h"] == "32", case["pad"])
    elif op == "quantize":
        n = case["width"]
        s.x = _rows(T, n, case["pad"], t, gen)
        s.gate = None if case["act"] == "none" else _rows(T, n, case["pad"], t, gen, 2.0)
        s.y = torch.empty_like(s.x)
        s.codes, s.scales = torch.empty((T, _up(n + case["pad"], 16)), dtype=torch.int8, device=_DEVICE), torch.empty((T,), device=_DEVICE)
    elif op == "w8":
        I = case["inputs"]
        s.codes = (torch.randn((T, _up(I + case["pad"], 16)), device=_DEVICE, generator=gen) * 35).round_().clamp_(-127, 127).to(torch.int8)
        s.scales = (0.5 + torch.rand((T,), device=_DEVICE, generator=gen)) / 35
        for _ in range(case["n"]):
            _weights(s, case["outputs"], I, gen)
        s.y = [torch.empty((T, case["outputs"]), dtype=torch.float32 if case["y"] == "32" else t, device=_DEVICE) for _ in range(case["n"])]
    else:
        n = case["width"]
        _norm_inputs(s, T, n, gen, case["post"])
        shapes = [(case["outputs"], n)] * 3 if op == "qkv" else [(case["wide"], n), (case["wide"], n), (n, case["wide"])]
        for O, I in shapes:
            _weights(s, O, I, gen)
        s.y = [torch.empty((T, O), dtype=t, device=_DEVICE) if op == "qkv" else _rows_for(T, O, t) for O, _ in shapes]
        s.codes, s.scales = torch.empty((T, _up(n, 16)), dtype=torch.int8, device=_DEVICE), torch.empty((T,), device=_DEVICE)
        if op == "mlp":
            s.wide_codes, s.wide_scales = torch.empty((T, _up(case["wide"], 16)), dtype=torch.int8, device=_DEVICE), torch.empty((T,), device=_DEVICE)
    return s


def _rows_for(T, O, t):
    """room for a product whose rows are read again 16 bytes at a time"""
    return torch.empty((T, _up(O, 8)), dtype=t, device=_DEVICE)


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2311_03285_amd import slora

    s.lib = slora
    dtype = slora.F16 if case["dtype"] == "f16" else slora.BF16
    s.dtype = dtype
    if case["op"] in ("norm", "qkv", "mlp"):
        flags = (slora.NORM_LAYER if case["kind"] == "layer" else 0) | (slora.NORM_POST if case["post"] else 0) | (slora.NORM_H32 if case.get("h") == "32" else 0)
        at = [None if v is None else v.data_ptr() for v in (s.post_w, s.post_b, s.pre_w, s.pre_b)]
        s.norm = slora.norm_init(case["width"], dtype, flags, _EPS, case.get("scale", 1.0), *at)
        s.close.append((slora.norm_destroy, s.norm))
    # weights are laid out once, when the model is loaded
    s.packed, s.handles = [], []
    for codes, scales in s.weights:
        O, I = codes.shape
        s.packed.append(torch.empty(slora.w8_bytes(O, I), dtype=torch.uint8, device=_DEVICE))
        s.handles.append(slora.w8_pack(O, I, dtype, codes.data_ptr(), scales.data_ptr(), s.packed[-1].data_ptr()))
        s.close.append((slora.w8_destroy, s.handles[-1]))
    s.act = {"none": slora.ACT_NONE, "silu": slora.ACT_SILU, "gelu": slora.ACT_GELU}[case.get("act", "none")]
    return s


# ---- one pass --------------------------------------------------------------------------------------
def _own_norm(s, x=None, codes=None):
    gate_stride = 0 if s.gate is None or s.gate.dim() == 1 else s.gate.stride(0)
    s.lib.norm_apply(s.norm, s.h.shape[0], s.h.data_ptr(), s.h.stride(0), s.block.data_ptr(), s.block.stride(0), None if s.gate is None else s.gate.data_ptr(), gate_stride,
                     s.h_out.data_ptr(), s.h_out.stride(0), None if x is None else x.data_ptr(), 0 if x is None else x.stride(0),
                     None if codes is None else codes.data_ptr(), 0 if codes is None else codes.stride(0), None if codes is None else s.scales.data_ptr())


def run(s):
    case = s.case
    T, op = case["tokens"], case["op"]
    if op == "norm":
        n = case["width"]
        if own:
            _own_norm(s, x=s.x)
        else:
            _plain_norm(s, x=s.x)
        return {"h": s.h_out[:, :n], "x": s.x[:, :n]}
    if op == "quantize":
        n, gated = case["width"], case["act"] != "none"
        if own:
            gate = (s.gate.data_ptr(), s.gate.stride(0)) if gated else (None, 0)
            if gated:
                s.lib.w8_quantize(T, n, s.dtype, s.act, s.x.data_ptr(), s.x.stride(0), *gate, y=s.y.data_ptr(), y_stride=s.y.stride(0))
            else:
                s.lib.w8_quantize(T, n, s.dtype, s.act, s.x.data_ptr(), s.x.stride(0), codes=s.codes.data_ptr(), codes_stride=s.codes.stride(0), scales=s.scales.data_ptr())
        elif gated:
            s.y[:, :n] = (_plain_act(case["act"], s.gate[:, :n].float()) * s.x[:, :n].float()).to(s.y.dtype)
        else:
            s.codes[:, :n], s.scales[:] = _plain_codes(s.x[:, :n].float())
        return {"y": s.y[:, :n]} if gated else {"codes": s.codes[:, :n], "scales": s.scales}
    if op == "w8":
        if own:
            product = s.lib.w8_matmul if case["y"] == "32" else s.lib.w8_matmul_y16
            product(s.handles, [s.codes.data_ptr()] * case["n"], [s.codes.stride(0)] * case["n"], [s.scales.data_ptr()] * case["n"], T, [y.data_ptr() for y in s.y],
                    [y.stride(0) for y in s.y])
        else:
            for k in range(case["n"]):
                _plain_product(s, k, s.codes, s.scales)
        return s.y
    if op == "qkv":
        if own:
            _own_norm(s, x=s.x, codes=s.codes)
            s.lib.w8_matmul_y16(s.handles, [s.codes.data_ptr()] * 3, [s.codes.stride(0)] * 3, [s.scales.data_ptr()] * 3, T, [y.data_ptr() for y in s.y],
                                [y.stride(0) for y in s.y])
        else:
            _plain_norm(s, x=s.x, codes=s.codes)
            for k in range(3):
                _plain_product(s, k, s.codes, s.scales)
        n = case["width"]
        return {"h": s.h_out[:, :n], "x": s.x[:, :n], "y": s.y}
    n, wide = case["width"], case["wide"]
    gate, up, down = s.y
    if own:
        _own_norm(s, codes=s.codes)
        s.lib.w8_matmul_y16(s.handles[:2], [s.codes.data_ptr()] * 2, [s.codes.stride(0)] * 2, [s.scales.data_ptr()] * 2, T, [gate.data_ptr(), up.data_ptr()],
                            [gate.stride(0), up.stride(0)])
        s.lib.w8_quantize(T, wide, s.dtype, s.act, up.data_ptr(), up.stride(0), gate.data_ptr(), gate.stride(0), codes=s.wide_codes.data_ptr(),
                          codes_stride=s.wide_codes.stride(0), scales=s.wide_scales.data_ptr())
        s.lib.w8_matmul_y16(s.handles[2:], [s.wide_codes.data_ptr()], [s.wide_codes.stride(0)], [s.wide_scales.data_ptr()], T, [down.data_ptr()], [down.stride(0)])
    else:
        _plain_norm(s, codes=s.codes)
        _plain_product(s, 0, s.codes, s.scales)
        _plain_product(s, 1, s.codes, s.scales)
        s.wide_codes[:, :wide], s.wide_scales[:] = _plain_codes(_plain_act(case["act"], gate[:, :wide].float()) * up[:, :wide].float())
        _plain_product(s, 2, s.wide_codes, s.wide_scales)
    return {"h": s.h_out[:, :n], "y": down[:, :n]}


# ---- plain forms, in 32 bits -------------------------------------------------------------------------
def _plain_normed(kind, v, w, b):
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + _EPS) * w.float()
    return v if b is None else v + b.float()


def _plain_norm(s, x=None, codes=None):
    case = s.case
    n = case["width"]
    b = s.block[:, :n].float()
    if case["post"]:
        b = _plain_normed(case["kind"], b, s.post_w, s.post_b)
    if s.gate is not None:
        b = b * s.gate[..., :n].float()
    h = s.h[:, :n].float() + case.get("scale", 1.0) * b
    s.h_out[:, :n] = h.to(s.h_out.dtype)
    v = _plain_normed(case["kind"], h, s.pre_w, s.pre_b)
    if x is not None:
        x[:, :n] = v.to(x.dtype)
    if codes is not None:
        codes[:, :n], s.scales[:] = _plain_codes(v)


def _plain_act(act, v):
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return 0.5 * v * (1 + torch.tanh(0.7978845608028654 * (v + 0.044715 * v * v * v)))


def _plain_codes(v):
    a = v.abs().amax(dim=1).clamp(min=_LEAST)
    return torch.round(v * (127 / a)[:, None]).to(torch.int8), a / 127


def _plain_product(s, k, codes, scales):
    """whole numbers below 2^24 are exact in 32 bits: sums of 1024 products are, and these are added as whole numbers"""
    w, by = s.weights[k]
    O, I = w.shape
    total = torch.zeros((codes.shape[0], O), dtype=torch.int32, device=_DEVICE)
    for i in range(0, I, 1024):
        total += torch.matmul(codes[:, i:min(i + 1024, I)].float(), w[:, i:i + 1024].float().t()).to(torch.int32)
    s.y[k][:, :O] = (total.float() * scales[:, None] * by).to(s.y[k].dtype)


# ---- the definition, in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    T, op, n = case["tokens"], case["op"], case.get("width")
    if op == "norm":
        h, x = _exact_norm(s)
        return {"h": h, "x": x}
    if op == "quantize":
        x = s.x[:, :n].double()
        if case["act"] != "none":
            return {"y": x * _exact_act(case["act"], s.gate[:, :n].double())}
        codes, scales = _exact_codes(x)
        return {"codes": codes.to(torch.int8), "scales": scales}
    if op == "w8":
        return [_exact_product(s.codes[:, :case["inputs"]].double(), s.scales, *w) for w in s.weights]
    h, x = _exact_norm(s)
    codes, scales = _exact_codes(x)
    if op == "qkv":
        return {"h": h, "x": x, "y": [_exact_product(codes, scales, *w) for w in s.weights]}
    # (gate and up are results of their own, in the 16-bit type)
    gate, up = (_exact_product(codes, scales, *w).to(_type(case)).double() for w in s.weights[:2])
    codes, scales = _exact_codes(up * _exact_act(case["act"], gate))
    return {"h": h, "y": _exact_product(codes, scales, *s.weights[2])}


def _exact_norm(s):
    case = s.case
    n = case["width"]

    def normed(v, weight, bias):
        if case["kind"] == "layer":
            spread, mean = torch.var_mean(v, dim=1, keepdim=True, correction=0)
            v = v - mean
        else:
            spread = v.square().sum(dim=1, keepdim=True) / n
        v = v * (spread + _EPS).rsqrt() * weight.double()
        return v if bias is None else v + bias.double()

    added = s.block[:, :n].double()
    if case["post"]:
        added = normed(added, s.post_w, s.post_b)
    if s.gate is not None:
        added = added * (s.gate.double() if s.gate.dim() == 1 else s.gate[:, :n].double())
    h = torch.add(s.h[:, :n].double(), added, alpha=case.get("scale", 1.0))
    return h, normed(h, s.pre_w, s.pre_b)


def _exact_act(act, v):
    if act == "silu":
        return v * torch.sigmoid(v)
    # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
    return v * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3))


def _exact_codes(v):
    """quotient and product of fp32 values, in 64 bits and rounded once, are what fp32 gives"""
    a = torch.linalg.vector_norm(v, ord=float("inf"), dim=1, keepdim=True).clamp(min=_LEAST)
    inverse = (127.0 / a.float().double()).float().double()
    return (v.float().double() * inverse).float().double().round(), (a / 127.0)[:, 0]


def _exact_product(codes, scales, weights, by):
    y = torch.empty((codes.shape[0], weights.shape[0]), dtype=torch.float64, device=_DEVICE)
    for o in range(0, weights.shape[0], 4096):
        y[:, o:o + 4096] = (codes @ weights[o:o + 4096].double().t().contiguous()) * by[o:o + 4096].double()
    return y * scales.double()[:, None]
