"""Norms, rows in 8 bits and products of 8-bit integers in 64 bits, with bounds on what 32-bit arithmetic may be off by.

E = 2^-24 is half a step of fp32.  A sum of a row is at most DEPTH additions deep: 8 elements of up to 9 pieces a lane, 6 steps over a
wavefront, 16 wavefronts, and the division by the width."""
import numpy as np
import torch

E = 2.0 ** -24
DEPTH = 72 + 6 + 16 + 1
HALF = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a step relative to the value
LEAST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # ... and below the normal numbers


def normed(v, e, w, c, layer, eps):
    """N(v; w, c) of rows that are known to +- e, and its bound"""
    n = v.shape[1]
    mean = v.mean(axis=1, keepdims=True) if layer else 0.0
    d = v - mean
    q = (d * d).mean(axis=1, keepdims=True) + eps
    r = 1 / np.sqrt(q)
    # the mean is off by its sum's roundings and by v's error; a difference by that, by v's own and one rounding
    off = (DEPTH * E * np.abs(v).mean(axis=1, keepdims=True) + e.mean(axis=1, keepdims=True) if layer else 0.0) + e + E * np.abs(d)
    # the mean square by its sum's, by the squares' and by those of the differences (first and second order), eps's addition; the root halves it
    rel = 0.5 * ((DEPTH + 3) * E + 2 * np.sqrt((off ** 2).mean(axis=1, keepdims=True)) * r + (off ** 2).mean(axis=1, keepdims=True) * r * r) + 3 * E
    x = d * r
    err = off * r * (1 + rel) + np.abs(x) * (rel + 2 * E)
    if w is not None:
        x, err = x * w, (err + E * np.abs(x)) * np.abs(w)
    if c is not None:
        x = x + c
        err = err + E * np.abs(x)
    return x, err


def norm(h, b, gate, scale, post, pre, layer, eps):
    """h', x and their bounds; post: None or (w, c), pre: (w, c)"""
    zero = np.zeros_like(h)
    if b is None:
        h2, e = h, zero
    else:
        v, e = (b, zero) if post is None else normed(b, zero, *post, layer, eps)
        if gate is not None:
            v, e = v * gate, (e + E * np.abs(v)) * np.abs(gate)
        h2 = h + scale * v
        e = abs(scale) * e + E * np.abs(h2)
    x, ex = normed(h2, e, *pre, layer, eps)
    return h2, e, x, ex


def within(got, ref, bound):
    """got (a tensor) is ref, off by at most the bound and one rounding to its type"""
    t = got.dtype
    g = got.double().cpu().numpy()
    slack = bound + HALF[t] * (np.abs(ref) + bound) + LEAST[t]
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(g - ref) <= slack)
    bad &= ~(np.isnan(g) & np.isnan(ref))
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(g - ref) / np.maximum(slack, 1e-300))), np.argwhere(bad)[:4].tolist())


def codes_of(v):
    """the definition, in fp32, of values that are fp32 numbers: (codes, scales)"""
    v = v.astype(np.float32)
    spoiled = ~np.isfinite(v).all(axis=1)
    with np.errstate(invalid="ignore"):
        a = np.maximum(np.where(spoiled, np.float32(1), np.abs(v).max(axis=1)), np.float32(2.0 ** -100)).astype(np.float32)
        c = np.rint(v * (np.float32(1) / a * np.float32(127))[:, None])
    return np.where(spoiled[:, None], 0, c).astype(np.int8), np.where(spoiled, np.float32(np.nan), a / np.float32(127))


def codes_within(codes, scales, ref, bound):
    """codes and scales stand for values that are ref to +- bound: a code is off by half of its scale, and by v's error in both places where v goes in"""
    c, s = codes.double().cpu().numpy(), scales.double().cpu().numpy()
    a = np.maximum(np.abs(ref).max(axis=1), 2.0 ** -100)
    ea = bound.max(axis=1)
    assert (np.abs(s - a / 127) <= ea / 127 + 2 * E * a / 127).all()
    # |v * inverse| <= 127 is off by four roundings (quotient, two products, scale) before the code is rounded
    slack = 0.5 * s[:, None] + bound + 127 * 5 * E * s[:, None]
    assert (np.abs(c * s[:, None] - ref) <= slack).all(), float((np.abs(c * s[:, None] - ref) - slack).max())
    assert np.abs(c).max() <= 127


def product(codes, scales, w, w_scales):
    ref = (codes.astype(np.float64) @ w.astype(np.float64).T) * scales[:, None].astype(np.float64) * w_scales.astype(np.float64)
    return ref, 3.001 * E * np.abs(ref)  # the sum to fp32, two products
