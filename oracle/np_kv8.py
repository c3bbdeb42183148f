"""Plain numpy fp64 oracle of the 8-bit KV cache and of the products with 4-bit weights: test infrastructure only.

A cache is kept per sequence, layer and head as codes [token, element] with exponents per block; attention, the weights that tokens
draw and eviction follow the definitions in include/slora.h token by token, in float64.
"""
from __future__ import annotations

import numpy as np

LOWEST, POISON = -60, 127


def exponent(values: np.ndarray) -> int:
    """least e >= -60 with |v| <= 127 * 2**e for all values; 127 if one is infinite or NaN"""
    if values.size == 0:
        return LOWEST
    if not np.isfinite(values).all():
        return POISON
    top = float(np.abs(values).max())
    e = LOWEST
    while top > 127.0 * 2.0 ** e:
        e += 1
    return e


def shifted(codes: np.ndarray, was: int, now: int) -> np.ndarray:
    if now == POISON:
        return np.zeros_like(codes)
    return np.rint(codes.astype(np.float64) * 2.0 ** (was - now)).astype(np.int8)


class Part:
    """K or V of one sequence, layer and head"""

    def __init__(self, D, N):
        self.D, self.N = D, N
        self.codes = np.zeros((0, D), np.int8)
        self.exps = []

    def append(self, rows):
        old, N = len(self.codes), self.N
        self.codes = np.concatenate([self.codes, np.zeros((len(rows), self.D), np.int8)])
        rows = rows.astype(np.float64)
        for b in range(old // N, -(-len(self.codes) // N) if len(rows) else 0):
            lo, hi = max(old, b * N), min(len(self.codes), (b + 1) * N)
            e = exponent(rows[lo - old:hi - old])
            if lo > b * N:
                was = self.exps[b]
                e = max(e, was)
                self.codes[b * N:lo] = shifted(self.codes[b * N:lo], was, e)
                self.exps[b] = e
            else:
                self.exps.append(e)
            if e != POISON:
                self.codes[lo:hi] = np.rint(rows[lo - old:hi - old] / 2.0 ** e).astype(np.int8)

    def cut(self, n):
        self.codes = self.codes[:n]
        self.exps = self.exps[:-(-n // self.N)]

    def values(self):
        unit = np.array([np.nan if e == POISON else 2.0 ** e for e in self.exps])[np.arange(len(self.codes)) // self.N]
        return self.codes * unit[:, None]

    def move(self, pairs, keep):
        """slots src -> dst, blocks of dst shifted to the largest exponent that comes"""
        codes, exps, N = self.codes.copy(), list(self.exps), self.N
        for b in sorted(set(d // N for _, d in pairs)):
            now = max([exps[b]] + [self.exps[s // N] for s, d in pairs if d // N == b])
            lo, hi = b * N, min((b + 1) * N, keep)
            codes[lo:hi] = shifted(self.codes[lo:hi], self.exps[b], now)
            exps[b] = now
        for s, d in pairs:
            codes[d] = shifted(self.codes[s], self.exps[s // N], exps[d // N])
        self.codes, self.exps = codes, exps


def attention(q, k, v, scale, visible):
    """q [rows, D], k and v [tokens, D], visible[r] tokens of row r: (out, probabilities, bound of the kernel's error before the last rounding)"""
    q, k, v = (a.astype(np.float64) for a in (q, k, v))
    out = np.zeros((len(q), v.shape[1]))
    p = np.zeros((len(q), len(k)))
    bound = np.zeros_like(out)
    p_rel = np.zeros(len(q))
    for r in range(len(q)):
        n = max(min(int(visible[r]), len(k)), 0)
        if n == 0:
            continue
        s = (k[:n] @ q[r]) * scale
        with np.errstate(invalid="ignore"):
            w = np.exp(s - s.max())
            p[r, :n] = w / w.sum()
            out[r] = p[r, :n] @ v[:n]
        # fp32 sums of D products and the exponent's argument, n terms of the sum: relative to each probability
        size = (np.abs(k[:n]) @ np.abs(q[r])).max() * abs(scale)
        delta = 2.0 ** -23 * (size * (k.shape[1] + 8) + n ** 0.5 + 64)
        p_rel[r] = 2 * delta
        share = p[r, :n] @ np.abs(v[:n])
        # probabilities rounded to 11 bits; below 2^-14 of the largest (times V's unit) to a multiple of 2^-24 of it
        unit = (p[r, :n, None] * np.abs(v[:n])).max() if n else 0.0
        bound[r] = (2.0 ** -11 + 2 * delta) * share + n * 2.0 ** -24 * 127 * unit * 2.0 ** -6
    return out, p, bound, p_rel


def evict(weights, pos, seen, keep, recent):
    """(moves [(src, dst)], weights and positions of the slots that stay)"""
    n = len(weights)
    recent = min(recent, keep)
    order = sorted(range(n), key=lambda i: (pos[i] < seen - recent, not np.isnan(weights[i]), -weights[i] if not np.isnan(weights[i]) else 0.0, i))
    stays = set(order[:keep])
    holes = [i for i in range(min(keep, n)) if i not in stays]
    src = [i for i in range(keep, n) if i in stays]
    moves = list(zip(src, holes))
    w, p = np.array(weights[:keep]), np.array(pos[:keep])
    for s, d in moves:
        w[d], p[d] = weights[s], pos[s]
    return moves, w, p


def w4(x, codes, scales, zeros, group):
    """x [T, inputs], codes [outputs, inputs], scales and zeros [outputs, groups]: (y, bound of an fp32 sum's error)"""
    g = np.arange(codes.shape[1]) // group
    w = (codes.astype(np.float64) - zeros.astype(np.float64)[:, g]) * scales.astype(np.float64)[:, g]
    # summed as c and as z: both sums' sizes count
    size = np.abs(x.astype(np.float64)) @ ((codes.astype(np.float64) + zeros.astype(np.float64)[:, g]) * np.abs(scales.astype(np.float64)[:, g])).T
    return x.astype(np.float64) @ w.T, size * 2.0 ** -23 * (4 + codes.shape[1] ** 0.5)
