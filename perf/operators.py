"""The attention side of a served layer: an 8-bit KV cache in the unified pool, and 4-bit base weights.

Four operators that a serving loop calls between the LoRA calls of a layer:

  append   new tokens' K and V are rounded to 8 bits into cache pages, with a power of two as scale
           for each block of tokens and head
  attend   attention over that cache, for prompts and for single tokens, if asked with the sums of
           attention weight that every cached token has drawn
  evict    of each head's cached tokens those of least accumulated weight make room: the tokens that
           stay move into their places, so that whole pages fall free
  w4       products of a few tokens with 4-bit weights that have a scale (and a zero) per group

A case of kind "attend" is one layer's append and attend, one of "evict" an eviction, one of "w4"
the products of up to eight matrices with the same tokens.

Layout of a cache page: a page of the pool (2*H bytes) belongs to one head and holds a block of
N = 8 * (H // (8 * D)) tokens in granules of eight.  A granule is 8*D bytes of K, [token][element],
and 8*D bytes of V, [element][token].  A code c stands for c * 2**e with the block's exponent e,
-60 <= e; e = 127 stands for a block that was given an infinity or NaN.
"""
from __future__ import annotations

import json
import math
import zlib

import numpy as np
import torch

own = False

_DEVICE = "cuda"
_LOWEST, _POISON = -60, 127  # exponents: the least one, and the one of a block with an infinity or NaN


def listed():
    cache = {"op": "attend", "H": 4096, "heads": 32, "kv_heads": 32, "head_dim": 128, "dtype": "f16", "decode": 0, "rows": 1,
             "prompts": 0, "chunk_lo": 0, "chunk_hi": 0, "shortest": 0, "longest": 0, "weights": False}
    evict = {"op": "evict", "H": 4096, "heads": 32, "kv_heads": 32, "head_dim": 128, "dtype": "f16", "seqs": 1, "shortest": 0,
             "longest": 0, "keep": 0, "recent": 0}
    w4 = {"op": "w4", "tokens": 1, "inputs": 4096, "outputs": 4096, "n": 1, "group": 128, "zeros": False, "dtype": "f16", "y": "f32"}

    def case(base, name, **kw):
        return {"name": name, **base, **kw}

    return [
        # a single interactive user: one token after a short conversation
        case(cache, "decode_1", decode=1, shortest=700, longest=700),
        # a decode batch with a head of K and V for every query head, whose cached tokens' weights are kept for eviction
        case(cache, "decode_weights", H=5120, heads=40, kv_heads=40, decode=24, shortest=200, longest=1500, weights=True),
        # a large decode batch of a wide model with shared heads, bfloat16
        case(cache, "decode_shared", H=8192, heads=64, kv_heads=8, dtype="bf16", decode=64, shortest=500, longest=8000),
        # two requests over very long documents: few rows, the work is along the cache
        case(cache, "decode_long", H=8192, heads=64, kv_heads=8, dtype="bf16", decode=2, shortest=90000, longest=131000),
        # uneven sizes: a width that leaves the end of a page unused, heads of 96, several drafted tokens per request
        case(cache, "decode_ragged", H=3080, heads=24, kv_heads=6, head_dim=96, dtype="bf16", decode=45, rows=3, shortest=0, longest=300),
        # one user's prompt on an empty cache
        case(cache, "prompt_1", prompts=1, chunk_lo=512, chunk_hi=512),
        # iteration-level batching: chunks of prompts with history beside decode tokens
        case(cache, "prompt_mixed", H=8192, heads=64, kv_heads=8, dtype="bf16", prompts=8, chunk_lo=128, chunk_hi=1024, decode=32,
             shortest=0, longest=4096),
        # caches at their budget, one token over it after each step
        case(evict, "evict_step", seqs=64, shortest=1025, longest=1025, keep=1024, recent=256),
        # long prompts cut down to an odd budget, shared heads
        case(evict, "evict_prompts", H=8192, heads=64, kv_heads=8, dtype="bf16", seqs=8, shortest=8000, longest=32000, keep=2041, recent=500),
        # the four attention projections of a single token
        case(w4, "w4_1", n=4),
        # a decode batch through the wide matrices of a layer, with zeros, in the model's 16-bit type
        case(w4, "w4_32", tokens=32, inputs=5120, outputs=20480, n=2, group=64, zeros=True, dtype="bf16", y="16"),
        # uneven sizes: inputs that end inside a tile, outputs that no tile divides, small groups, drafted tokens
        case(w4, "w4_ragged", tokens=67, inputs=3080, outputs=5003, n=3, group=32, zeros=True),
    ]


def draw(rng):
    """One more case of the kinds and ranges above."""

    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    most = [work(c) for c in listed()]
    top = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["attend", "attend", "attend", "evict", "w4"])
        dtype = rng.choice(["f16", "bf16"])
        if op == "w4":
            group = rng.choice([32, 64, 128, 128, 32 * spread(1, 16)])
            c = {"op": op, "tokens": spread(1, 256), "inputs": rng.choice([1024, 2048, 4096, 5120, 8192, 16384, 8 * spread(8, 2048)]),
                 "outputs": rng.choice([1024, 4096, 5120, 8192, 16384, spread(1, 20480)]), "n": rng.choice([1, 1, 2, 3, 4, 8]),
                 "group": group, "zeros": rng.random() < 0.5, "dtype": dtype, "y": rng.choice(["f32", "16"])}
        else:
            D = rng.choice([64, 128, 128, 128, 96, 256, 32])
            kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
            shared = rng.choice([1, 1, 2, 4, 5, 8, 16])
            # a page holds at least one granule of eight tokens
            H = max(8 * D, min(8192, kv * shared * D)) if rng.random() < 0.7 else 8 * spread(D, 1024)
            c = {"op": op, "H": H, "heads": kv * shared, "kv_heads": kv, "head_dim": D, "dtype": dtype}
            if op == "evict":
                longest = spread(16, 32000)
                shortest = spread(1, longest)
                keep = spread(1, longest)
                c.update(seqs=spread(1, 64), shortest=shortest, longest=longest, keep=keep, recent=rng.choice([0, keep, int(rng.random() * keep)]))
            else:
                c.update(decode=0, rows=1, prompts=0, chunk_lo=0, chunk_hi=0, shortest=0, longest=0, weights=rng.random() < 0.3)
                kind = rng.choice(["decode", "decode", "decode", "prompt", "mixed"])
                c["longest"] = spread(1, 131000) if kind == "decode" else rng.choice([0, spread(1, 16000)])
                c["shortest"] = int(rng.random() * c["longest"]) if rng.random() < 0.7 else 0
                if kind != "prompt":
                    c["decode"] = spread(1, 128)
                    c["rows"] = rng.choice([1, 1, 1, 2, 4, 9])
                if kind != "decode":
                    c["prompts"] = spread(1, 12)
                    c["chunk_hi"] = spread(2, 2048)
                    c["chunk_lo"] = spread(1, c["chunk_hi"])
        w = work(c)
        if w["bytes"] <= top["bytes"] and w["flops"] <= top["flops"] and _held(c) <= 4 << 30:
            return c


# ---- what a case means ---------------------------------------------------------------------------
def _rng(case):
    return np.random.RandomState(zlib.crc32(json.dumps({k: v for k, v in case.items() if k != "name"}, sort_keys=True).encode()))


def _block(case):
    """tokens per page"""
    return 8 * (case["H"] // (8 * case["head_dim"]))


def _sequences(case):
    """[(tokens in the cache before the call, new tokens)] of every sequence: from the case alone."""
    rng = _rng(case)
    if case["op"] == "evict":
        return [(int(v), 0) for v in rng.randint(case["shortest"], case["longest"] + 1, case["seqs"])]
    n = case["prompts"] + case["decode"]
    old = [int(v) for v in rng.randint(case["shortest"], case["longest"] + 1, n)]
    new = [int(v) for v in rng.randint(case["chunk_lo"], case["chunk_hi"] + 1, case["prompts"])]
    new += [int(v) for v in rng.randint(1, case["rows"] + 1, case["decode"])]
    return list(zip(old, new))


def _held(case):
    """bytes of cache, or of weights"""
    if case["op"] == "w4":
        return case["n"] * case["outputs"] * case["inputs"] // 2
    return sum(2 * case["kv_heads"] * case["head_dim"] * (old + new) for old, new in _sequences(case))


def work(case):
    """attend: the codes of every cached token and the new rows once; evict: weights and positions once, the expected
    number of moved tokens read and written; w4: codes, scales, zeros, x and y once."""
    if case["op"] == "w4":
        groups = -(-case["inputs"] // case["group"])
        weight = case["outputs"] * (case["inputs"] // 2 + groups * (3 if case["zeros"] else 2))
        y = case["tokens"] * case["outputs"] * (4 if case["y"] == "f32" else 2)
        return {"bytes": case["n"] * (weight + y) + case["tokens"] * case["inputs"] * 2,
                "flops": 2 * case["n"] * case["tokens"] * case["outputs"] * case["inputs"]}
    D, kv, heads = case["head_dim"], case["kv_heads"], case["heads"]
    if case["op"] == "evict":
        total, ranked = 0, 0
        for size, _ in _sequences(case):
            keep, recent = min(case["keep"], size), min(case["recent"], case["keep"], size)
            moved = min(size - keep, recent + (keep - recent) * max(size - recent - keep, 0) / max(size - recent, 1))
            total += kv * (8 * size + 8 * keep + 4 * D * moved)
            ranked += kv * size
        return {"bytes": int(total), "flops": ranked}
    cached, rows, flops = 0, 0, 0
    for old, new in _sequences(case):
        cached += old + new
        rows += new
        flops += 4 * D * heads * (new * old + new * (new + 1) // 2)
    moved = 2 * kv * D * cached + 2 * rows * D * (2 * heads + 2 * kv) + 2 * kv * -(-cached // _block(case))
    if case["weights"]:
        moved += 8 * kv * cached
    return {"bytes": moved, "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------------
def _type(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _codes(n, gen, spread=32.0):
    out = torch.empty(n, dtype=torch.int8, device=_DEVICE)
    step = 1 << 26
    for at in range(0, n, step):
        out[at:at + step] = (torch.randn(min(step, n - at), device=_DEVICE, generator=gen) * spread).round_().clamp_(-127, 127)
    return out


class _State:
    def __init__(self, case):
        self.case = case
        self.close = []

    def __del__(self):
        for end, handle in self.close:
            end(handle)


def _cache_inputs(s, case, seed):
    """A pool with a cache for every sequence, the batch's rows, and what eviction goes by."""
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 32))
    H, D, kv, heads, N = case["H"], case["head_dim"], case["kv_heads"], case["heads"], _block(case)
    s.sequences = _sequences(case)
    s.n = len(s.sequences)
    blocks = [-(-(old + new) // N) for old, new in s.sequences]
    s.max_tokens = max(1, max(old + new for old, new in s.sequences))
    s.max_blocks = -(-s.max_tokens // N)
    used = sum(blocks) * kv
    n_pages = used + used // 4 + 8
    # pages anywhere in a pool that others use as well
    place = rng.permutation(n_pages)[:used].astype(np.int32)
    s.page_list, s.pages, at = place, [], 0
    for b in blocks:
        s.pages.append(torch.from_numpy(place[at:at + b * kv].astype(np.int64).reshape(b, kv)).to(_DEVICE))
        at += b * kv
    s.pool = _codes(n_pages * 2 * H, gen).view(n_pages, 2 * H)
    # K and V of order one: codes spread over 32 of 127, blocks of different exponents
    s.exps = torch.randint(-6, -3, (s.n, s.max_blocks, 1, kv, 2), dtype=torch.int8, device=_DEVICE, generator=gen)
    s.first = np.concatenate([[0], np.cumsum([new for _, new in s.sequences])])
    rows = int(s.first[-1])
    s.seen = [old + new for old, new in s.sequences]
    if case["op"] == "evict":
        # few tokens draw much weight, as attention's do; equal sums occur (tokens that drew nothing)
        w = torch.exp(2 * torch.randn((s.n, kv, s.max_tokens), device=_DEVICE, generator=gen))
        w[torch.rand(w.shape, device=_DEVICE, generator=gen) < 0.1] = 0.0
        s.weights = w
        s.weights_out = torch.zeros_like(w)
        # slots hold tokens in order, apart from those that took a place in earlier evictions
        s.pos = torch.arange(s.max_tokens, dtype=torch.int32, device=_DEVICE).expand(s.n, kv, -1).contiguous()
        for i, (size, _) in enumerate(s.sequences):
            half = size // 2
            order = torch.rand((kv, half), device=_DEVICE, generator=gen).argsort(dim=1)
            s.pos[i, :, :half] = order.to(torch.int32)
        s.pos_out = torch.zeros_like(s.pos)
        return
    # what the projection of q, k and v leaves: one row per token
    s.qkv = torch.randn((rows, (heads + 2 * kv) * D), device=_DEVICE, generator=gen)
    s.qkv[:, :heads * D] *= 2
    s.qkv = s.qkv.to(_type(case))
    s.out = torch.empty((rows, heads * D), dtype=_type(case), device=_DEVICE)
    s.scale = 1.0 / math.sqrt(D)
    if case["weights"]:
        s.weights = torch.rand((s.n, kv, s.max_tokens), device=_DEVICE, generator=gen)
        s.weights_out = torch.zeros_like(s.weights)
        s.pos = torch.arange(s.max_tokens, dtype=torch.int32, device=_DEVICE).expand(s.n, kv, -1).contiguous()


def _w4_inputs(s, case, seed):
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(seed)
    I, O, groups = case["inputs"], case["outputs"], -(-case["inputs"] // case["group"])
    s.codes, s.scales, s.zeros, s.y = [], [], [], []
    for _ in range(case["n"]):
        # two codes a byte, the first in the low four bits; around the zero as rounding normal weights leaves them
        c = (torch.randn((O, I), device=_DEVICE, generator=gen) * 2.6 + 8).round_().clamp_(0, 15).to(torch.uint8)
        s.codes.append(c[:, 0::2] | (c[:, 1::2] << 4))
        del c
        s.scales.append(((0.5 + torch.rand((O, groups), device=_DEVICE, generator=gen)) / (2.6 * math.sqrt(I))).to(_type(case)))
        s.zeros.append(torch.randint(6, 11, (O, groups), dtype=torch.uint8, device=_DEVICE, generator=gen) if case["zeros"] else None)
        s.y.append(torch.empty((case["tokens"], O), dtype=torch.float32 if case["y"] == "f32" else _type(case), device=_DEVICE))
    s.x = torch.randn((case["tokens"], I), device=_DEVICE, generator=gen).to(_type(case))


def prepare(case, seed):
    s = _State(case)
    if case["op"] == "w4":
        _w4_inputs(s, case, seed)
    else:
        _cache_inputs(s, case, seed)
    if not own:
        return s
    from paper_2311_03285_amd import slora

    s.lib = slora
    dtype = slora.F16 if case["dtype"] == "f16" else slora.BF16
    if case["op"] == "w4":
        # weights are laid out once, when the model is loaded
        s.packed = [torch.empty(slora.w4_bytes(case["outputs"], case["inputs"], case["group"]), dtype=torch.uint8, device=_DEVICE)
                    for _ in range(case["n"])]
        s.handles = []
        for k in range(case["n"]):
            s.handles.append(slora.w4_pack(case["outputs"], case["inputs"], case["group"], dtype, s.codes[k].data_ptr(), s.scales[k].data_ptr(),
                                           s.zeros[k].data_ptr() if case["zeros"] else None, s.packed[k].data_ptr()))
            s.close.insert(0, (slora.w4_destroy, s.handles[k]))
        s.xs = [s.x.data_ptr()] * case["n"]
        s.ys = [y.data_ptr() for y in s.y]
        return s
    pool = slora.pool_init(case["H"], s.pool.shape[0], dtype, s.pool.data_ptr(), 1, 0)
    s.close.insert(0, (slora.pool_destroy, pool))
    cache = slora.kv8_init(pool, 1, case["heads"], case["kv_heads"], case["head_dim"], s.n, s.max_tokens, s.exps.data_ptr())
    s.close.insert(0, (slora.kv8_destroy, cache))
    seqs = np.arange(s.n, dtype=np.int32)
    slora.kv8_extend(cache, seqs, [old + new for old, new in s.sequences], s.page_list)
    keep = [min(case["keep"], size) for size, _ in s.sequences] if case["op"] == "evict" else None
    s.batch = slora.kv8_batch_plan(cache, seqs, [new for _, new in s.sequences], keep)
    s.close.insert(0, (slora.kv8_batch_destroy, s.batch))
    return s


# ---- one pass --------------------------------------------------------------------------------------
def run(s):
    case = s.case
    if case["op"] == "w4":
        if own:
            (s.lib.w4_matmul if case["y"] == "f32" else s.lib.w4_matmul_y16)(s.handles, s.xs, case["tokens"], s.ys)
        else:
            for k in range(case["n"]):
                _plain_w4(s, k)
        return s.y
    if case["op"] == "evict":
        if own:
            s.lib.kv8_evict(s.batch, 0, case["recent"], s.weights.data_ptr(), s.weights_out.data_ptr(), s.pos.data_ptr(), s.pos_out.data_ptr())
        else:
            for i in range(s.n):
                _plain_evict(s, i)
        return {"pool": s.pool, "exps": s.exps, "weights": s.weights_out, "pos": s.pos_out}
    if own:
        heads, kv, D = case["heads"], case["kv_heads"], case["head_dim"]
        q, width = s.qkv.data_ptr(), (heads + 2 * kv) * D
        k = q + heads * D * 2
        s.lib.kv8_append(s.batch, 0, k, width, k + kv * D * 2, width)
        weights = (s.weights.data_ptr(), s.weights_out.data_ptr(), s.pos.data_ptr()) if case["weights"] else None
        s.lib.kv8_attend(s.batch, 0, q, width, s.out.data_ptr(), heads * D, s.scale, True, weights)
    else:
        for i in range(s.n):
            _plain_append(s, i)
            _plain_attend(s, i)
    out = {"out": s.out, "pool": s.pool, "exps": s.exps}
    if case["weights"]:
        out.update(weights=s.weights_out, pos=s.pos)
    return out


# ---- plain forms, in 32 bits -------------------------------------------------------------------------
def _two(e):
    """2**e in float32, from the bits; NaN for the exponent of a block that holds an infinity or NaN"""
    e = e.to(torch.int32)
    p = ((e.clamp(-126, 126) + 127) << 23).view(torch.float32)
    return torch.where(e == _POISON, torch.full_like(p, math.nan), p)


def _exponent(amax):
    """least e >= -60 with amax <= 127 * 2**e"""
    bits = amax.view(torch.int32)
    e = (((bits - 0x7E0001) >> 23) - 132).clamp(min=_LOWEST)
    return torch.where(torch.isfinite(amax), e, torch.full_like(e, _POISON))


def _rounded(values, e):
    """codes of values (or of other codes) in units of 2**e; those of a poisoned block are 0"""
    c = torch.round(values * _two(-e.clamp(max=126)))
    return torch.where((e == _POISON) | ~torch.isfinite(c), torch.zeros_like(c), c).to(torch.int8)


def _fetch(s, i, b0, b1):
    """K and V codes of blocks [b0, b1) of sequence i: [head][token][element]"""
    case = s.case
    D, kv, N = case["head_dim"], case["kv_heads"], _block(case)
    g = s.pool[s.pages[i][b0:b1]][:, :, :N * 2 * D].view(b1 - b0, kv, N // 8, 2, 8 * D)
    k = g[:, :, :, 0].reshape(b1 - b0, kv, N, D).transpose(0, 1).reshape(kv, -1, D)
    v = g[:, :, :, 1].reshape(b1 - b0, kv, N // 8, D, 8).transpose(3, 4).reshape(b1 - b0, kv, N, D).transpose(0, 1).reshape(kv, -1, D)
    return k, v


def _store(s, i, b0, b1, k, v):
    case = s.case
    D, kv, N = case["head_dim"], case["kv_heads"], _block(case)
    n = b1 - b0
    k = k.reshape(kv, n, N, D).transpose(0, 1).reshape(n, kv, N // 8, 1, 8 * D)
    v = v.reshape(kv, n, N, D).transpose(0, 1).reshape(n, kv, N // 8, 8, D).transpose(3, 4).reshape(n, kv, N // 8, 1, 8 * D)
    page = s.pool[s.pages[i][b0:b1]]
    page[:, :, :N * 2 * D] = torch.cat([k, v], dim=3).reshape(n, kv, N * 2 * D)
    s.pool[s.pages[i][b0:b1]] = page


def _plain_append(s, i):
    case = s.case
    D, kv, heads, N = case["head_dim"], case["kv_heads"], case["heads"], _block(case)
    old, new = s.sequences[i]
    if new == 0:
        return
    b0, b1 = old // N, -(-(old + new) // N)
    rows = s.qkv[int(s.first[i]):int(s.first[i + 1]), heads * D:].float().view(new, 2, kv, D).permute(1, 2, 0, 3)
    at = old - b0 * N
    done = []
    for which, codes in enumerate(_fetch(s, i, b0, b1)):
        fresh = torch.zeros((kv, (b1 - b0) * N, D), device=_DEVICE)
        fresh[:, at:at + new] = rows[which]
        amax = fresh.view(kv, b1 - b0, N * D).abs().amax(dim=2)
        before = s.exps[i, b0:b1, 0, :, which].t().to(torch.int32).clone()
        before[:, 1 if at else 0:] = _LOWEST  # blocks that begin with new tokens
        e = torch.maximum(_exponent(amax), before)
        per = e.repeat_interleave(N, dim=1)[:, :, None]
        was = before.repeat_interleave(N, dim=1)[:, :at, None]
        shift = (per[:, :at] - was).clamp(max=100)
        kept = torch.round(codes[:, :at].float() * _two(-shift)).to(torch.int8)
        codes = codes.clone()
        codes[:, :at] = torch.where(per[:, :at] == _POISON, torch.zeros_like(kept), kept)
        codes[:, at:at + new] = _rounded(fresh[:, at:at + new], per[:, at:at + new].expand(-1, -1, D))
        s.exps[i, b0:b1, 0, :, which] = e.t().to(torch.int8)
        done.append(codes)
    _store(s, i, b0, b1, *done)


def _plain_attend(s, i):
    case = s.case
    D, kv, heads, N = case["head_dim"], case["kv_heads"], case["heads"], _block(case)
    old, new = s.sequences[i]
    size, r0, r1 = old + new, int(s.first[i]), int(s.first[i + 1])
    if new == 0:
        return
    blocks = -(-size // N)
    codes = _fetch(s, i, 0, blocks)
    k, v = (codes[w][:, :size].float() * _two(s.exps[i, :blocks, 0, :, w]).t().repeat_interleave(N, dim=1)[:, :size, None] for w in (0, 1))
    q = s.qkv[r0:r1, :heads * D].float().view(new, kv, heads // kv, D).permute(1, 2, 0, 3).reshape(kv, -1, D)
    score = torch.matmul(q, k.transpose(1, 2).contiguous()).view(kv, heads // kv, new, size) * s.scale
    hidden = torch.arange(size, device=_DEVICE)[None, :] > old + torch.arange(new, device=_DEVICE)[:, None]
    score = score.masked_fill(hidden, -math.inf)
    p = torch.exp(score - score.amax(dim=3, keepdim=True))
    p = p / p.sum(dim=3, keepdim=True)
    o = torch.matmul(p.view(kv, -1, size), v)
    s.out[r0:r1] = o.view(kv, heads // kv, new, D).permute(2, 0, 1, 3).reshape(new, heads * D).to(s.out.dtype)
    if case["weights"]:
        total = p.sum(dim=(1, 2))
        total[:, :old] += s.weights[i, :, :old]
        s.weights_out[i, :, :size] = total
        s.pos[i, :, old:size] = torch.arange(s.seen[i] - new, s.seen[i], dtype=torch.int32, device=_DEVICE)


def _plain_evict(s, i):
    case = s.case
    D, kv, N = case["head_dim"], case["kv_heads"], _block(case)
    size = s.sequences[i][0]
    keep = min(case["keep"], size)
    w, pos = s.weights[i, :, :size], s.pos[i, :, :size]
    # recent tokens, then by weight, equal weights by slot
    order = torch.sort(w, dim=1, descending=True, stable=True).indices
    recent = (pos >= s.seen[i] - case["recent"]).gather(1, order)
    order = order.gather(1, torch.sort((~recent).to(torch.uint8), dim=1, stable=True).indices)
    kept = torch.zeros((kv, size), dtype=torch.bool, device=_DEVICE)
    kept.scatter_(1, order[:, :keep], True)
    # as many tokens stay behind the budget as there are places before it; in order, head by head
    head, place = (~kept[:, :keep]).nonzero(as_tuple=True)
    source = kept[:, keep:].nonzero(as_tuple=True)[1] + keep
    s.weights_out[i, :, :keep] = w[:, :keep]
    s.weights_out[i, head, place] = w[head, source]
    s.pos_out[i, :, :keep] = pos[:, :keep]
    s.pos_out[i, head, place] = pos[head, source]
    if size <= keep or keep == 0:
        return
    done, blocks = [], -(-keep // N)
    for which, codes in enumerate(_fetch(s, i, 0, s.pages[i].shape[0])):
        before = s.exps[i, :, 0, :, which].t().to(torch.int32)
        came = before[head, source // N]
        e = before[:, :blocks].clone().reshape(-1)
        e.scatter_reduce_(0, head * blocks + place // N, came, "amax")
        e = e.view(kv, blocks)
        stay = codes[:, :blocks * N].clone()
        shift = (e - before[:, :blocks]).clamp(max=100).repeat_interleave(N, dim=1)[:, :keep, None]
        poisoned = (e == _POISON).repeat_interleave(N, dim=1)[:, :keep, None]
        stay[:, :keep] = torch.where(poisoned, torch.zeros_like(stay[:, :keep]), torch.round(stay[:, :keep].float() * _two(-shift)).to(torch.int8))
        to = e[head, place // N]
        moved = torch.round(codes[head, source].float() * _two(-(to - came).clamp(max=100))[:, None]).to(torch.int8)
        stay[head, place] = torch.where((to == _POISON)[:, None], torch.zeros_like(moved), moved)
        s.exps[i, :blocks, 0, :, which] = e.t().to(torch.int8)
        done.append(stay)
    _store(s, i, 0, blocks, *done)


def _plain_w4(s, k):
    case = s.case
    I, O = case["inputs"], case["outputs"]
    c = torch.stack([s.codes[k] & 15, s.codes[k] >> 4], dim=2).view(O, I).float()
    zero = s.zeros[k].float() if case["zeros"] else torch.full((O, s.scales[k].shape[1]), 8.0, device=_DEVICE)
    each = case["group"]
    w = (c - zero.repeat_interleave(each, dim=1)[:, :I]) * s.scales[k].float().repeat_interleave(each, dim=1)[:, :I]
    s.y[k].copy_(torch.matmul(s.x.float(), w.t()))


# ---- the definition, in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    s = _State(case)
    if case["op"] == "w4":
        _w4_inputs(s, case, seed)
        return [_exact_w4(s, k) for k in range(case["n"])]
    _cache_inputs(s, case, seed)
    return _exact_evict(s) if case["op"] == "evict" else _exact_attend(s)


def _power(e):
    """2**e in float64, exactly (values rounded to 8 bits are often halfway between two codes)"""
    return torch.tensor([2.0 ** k for k in range(-260, 261)], dtype=torch.float64, device=_DEVICE)[e.long() + 260]


def _exact_w4(s, k):
    case = s.case
    I, O = case["inputs"], case["outputs"]
    group = torch.arange(I, device=_DEVICE) // case["group"]
    y = torch.empty((case["tokens"], O), dtype=torch.float64, device=_DEVICE)
    for o in range(0, O, 2048):
        byte = s.codes[k][o:o + 2048].long()
        w = torch.empty((byte.shape[0], I), dtype=torch.float64, device=_DEVICE)
        w[:, 0::2], w[:, 1::2] = (byte % 16).double(), (byte // 16).double()
        w -= s.zeros[k][o:o + 2048].double()[:, group] if case["zeros"] else 8.0
        w *= s.scales[k][o:o + 2048].double()[:, group]
        y[:, o:o + 2048] = s.x.double() @ w.t().contiguous()
    return y


def _addresses(s, i, head, token, which):
    """flat index in the pool of the D codes of K (which = 0) or V (1) of tokens `token` of a head"""
    case = s.case
    D, N = case["head_dim"], _block(case)
    page = s.pages[i][token // N, head]
    slot = token % N
    base = page * 2 * case["H"] + (slot // 8) * 16 * D
    d = torch.arange(D, device=_DEVICE)
    if which == 0:
        return base[:, None] + (slot % 8)[:, None] * D + d[None, :]
    return base[:, None] + 8 * D + d[None, :] * 8 + (slot % 8)[:, None]


def _exact_attend(s):
    case = s.case
    D, kv, heads, N = case["head_dim"], case["kv_heads"], case["heads"], _block(case)
    shared = heads // kv
    pool, exps = s.pool.clone().view(-1), s.exps.clone()
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=_DEVICE)
    weights = s.weights_out.double() if case["weights"] else None
    pos = s.pos.clone() if case["weights"] else None
    for i, (old, new) in enumerate(s.sequences):
        size, r0 = old + new, int(s.first[i])
        if new == 0:
            continue
        x = s.qkv[r0:r0 + new].double()
        token = torch.arange(size, device=_DEVICE)
        for h in range(kv):
            both = []
            for which in (0, 1):
                rows = x[:, (heads + which * kv + h) * D:][:, :D]
                at = _addresses(s, i, h, token, which)
                code = pool[at].double()
                size_of = rows.abs().amax(dim=1)
                m, e = torch.frexp(size_of)  # rows <= m * 2**e, m < 1: 127 * 2**(e - 7) holds it up to m = 127/128
                need = torch.where(size_of > 0, torch.where(m <= 127 / 128, e - 7, e - 6), torch.full_like(e, _LOWEST)).clamp(min=_LOWEST)
                block = token // N
                first = old // N
                was = exps[i, :, 0, h, which].long()
                now = was.clone()
                start = first + (1 if old % N else 0)
                now[start:-(-size // N)] = _LOWEST
                now.scatter_reduce_(0, block[old:], need.long(), "amax")
                factor = _power(was - now)[block]
                part = slice(first * N, old)
                code[part] = torch.round(code[part] * factor[part, None])
                unit = _power(now)[block][:, None]
                code[old:] = torch.round(rows / unit[old:])
                pool[at[first * N:]] = code[first * N:].to(torch.int8)
                exps[i, :, 0, h, which] = now.to(torch.int8)
                both.append(code * unit)
            k, v = both
            q = x[:, h * shared * D:(h + 1) * shared * D].reshape(new * shared, D)
            score = (q @ k.t().contiguous()).view(new, shared, size) * s.scale
            score.masked_fill_((token[None, :] > old + torch.arange(new, device=_DEVICE)[:, None])[:, None, :], -math.inf)
            p = torch.softmax(score, dim=2)
            out[r0:r0 + new, h * shared * D:(h + 1) * shared * D] = (p.view(-1, size) @ v).view(new, shared * D)
            if weights is not None:
                weights[i, h, :size] = p.sum(dim=(0, 1))
                weights[i, h, :old] += s.weights[i, h, :old].double()
                pos[i, h, old:size] = token[old:].to(torch.int32)
    result = {"out": out, "pool": pool.view(s.pool.shape), "exps": exps}
    if weights is not None:
        result.update(weights=weights, pos=pos)
    return result


def _exact_evict(s):
    case = s.case
    N, kv = _block(case), case["kv_heads"]
    pool, exps = s.pool.clone().view(-1), s.exps.clone()
    weights, pos_out = s.weights_out.double(), s.pos_out.clone()
    all_w, all_pos = s.weights.cpu().numpy(), s.pos.cpu().numpy()
    for i, (size, _) in enumerate(s.sequences):
        keep = min(case["keep"], size)
        for h in range(kv):
            w, pos = all_w[i, h, :size].astype(np.float64), all_pos[i, h, :size]
            rank = np.lexsort((np.arange(size), -w, pos < s.seen[i] - case["recent"]))
            stays = np.zeros(size, dtype=bool)
            stays[rank[:keep]] = True
            slot = np.arange(keep)
            slot[~stays[:keep]] = np.nonzero(stays[keep:])[0] + keep
            weights[i, h, :keep] = torch.from_numpy(w[slot]).to(_DEVICE)
            pos_out[i, h, :keep] = torch.from_numpy(pos[slot]).to(_DEVICE)
            if keep == size or keep == 0:
                continue
            source = torch.from_numpy(slot).to(_DEVICE)
            place = torch.arange(keep, device=_DEVICE)
            for which in (0, 1):
                was = exps[i, :, 0, h, which].long()
                now = was.clone()
                now.scatter_reduce_(0, place // N, was[source // N], "amax")
                change = _power(was[source // N] - now[place // N])
                moved = torch.round(s.pool.view(-1)[_addresses(s, i, h, source, which)].double() * change[:, None])
                pool[_addresses(s, i, h, place, which)] = moved.to(torch.int8)
                exps[i, :, 0, h, which] = now.to(torch.int8)
    return {"pool": pool.view(s.pool.shape), "exps": exps, "weights": weights, "pos": pos_out}
