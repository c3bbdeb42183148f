"""A KV cache on the GPU beside the oracle's: what the tests of the 8-bit cache share."""
import numpy as np
import torch

from oracle import np_kv8
from paper_2311_03285_amd import slora

DTYPES = {"f16": (slora.F16, torch.float16), "bf16": (slora.BF16, torch.bfloat16)}


class Twin:
    """The library's cache and the oracle's, fed the same rows."""

    def __init__(self, H, D, kv, G, dtype="f16", layers=1, max_seqs=4, max_tokens=600, n_pages=None, fill=None, seed=0):
        self.H, self.D, self.kv, self.G, self.layers, self.max_tokens, self.max_seqs = H, D, kv, G, layers, max_tokens, max_seqs
        self.lib_dtype, self.dtype = DTYPES[dtype]
        self.N = 8 * (H // (8 * D))
        self.blocks = slora.kv8_block_count(H, D, max_tokens)
        self.rng = np.random.default_rng(seed)
        n_pages = n_pages or max_seqs * self.blocks * layers * kv + 3
        # bytes that no token has written are any bytes
        self.pool = torch.from_numpy(self.rng.integers(-128, 128, (n_pages, 2 * H), dtype=np.int8)).cuda() if fill is None else fill(n_pages, 2 * H)
        self.exps = torch.full((max_seqs, self.blocks, layers, kv, 2), 77, dtype=torch.int8, device="cuda")
        self.lib_pool = slora.pool_init(H, n_pages, self.lib_dtype, self.pool.data_ptr(), 1, 0)
        self.cache = slora.kv8_init(self.lib_pool, layers, kv * G, kv, D, max_seqs, max_tokens, self.exps.data_ptr())
        self.part = {(s, l, h, w): np_kv8.Part(D, self.N) for s in range(max_seqs) for l in range(layers) for h in range(kv) for w in (0, 1)}
        self.pages = {s: np.zeros((0, layers, kv), np.int32) for s in range(max_seqs)}
        self.len = [0] * max_seqs
        self.seen = [0] * max_seqs
        self.free = self.rng.permutation(n_pages).astype(np.int32).tolist()
        self.batches = []

    def extend(self, seqs, tokens):
        new = []
        for s, t in zip(seqs, tokens):
            b = -(-(self.len[s] + t) // self.N) - -(-self.len[s] // self.N)
            mine = np.array([self.free.pop() for _ in range(b * self.layers * self.kv)], np.int32).reshape(b, self.layers, self.kv)
            self.pages[s] = np.concatenate([self.pages[s], mine])
            new.append(mine.reshape(-1))
            self.len[s] += t
            self.seen[s] += t
        slora.kv8_extend(self.cache, seqs, tokens, np.concatenate(new) if new else np.zeros(0, np.int32))

    def truncate(self, seqs, lengths, evicted=False):
        slora.kv8_truncate(self.cache, seqs, lengths, evicted)
        for s, n in zip(seqs, lengths):
            stay = -(-n // self.N)
            self.free += self.pages[s][stay:].reshape(-1).tolist()
            self.pages[s] = self.pages[s][:stay]
            if not evicted:
                self.seen[s] -= self.len[s] - n
            self.len[s] = n
            if n == 0:
                self.seen[s] = 0
            for l in range(self.layers):
                for h in range(self.kv):
                    for w in (0, 1):
                        self.part[s, l, h, w].cut(n)

    def plan(self, seqs, rows, keep=None):
        self.batches.append(slora.kv8_batch_plan(self.cache, seqs, rows, keep))
        return self.batches[-1]

    def rows(self, n, size=1.0):
        """n tokens' K and V, as the device's 16-bit tensor [n, 2, kv, D]"""
        return (torch.from_numpy(self.rng.standard_normal((n, 2, self.kv, self.D)) * size)).to(self.dtype).cuda()

    def append(self, batch, layer, seqs, counts, rows, oracle=True):
        at = rows.data_ptr()
        width = self.kv * self.D
        slora.kv8_append(batch, layer, at, 2 * width, at + 2 * width, 2 * width)
        host, r = rows.double().cpu().numpy(), 0
        for s, n in zip(seqs, counts):
            for h in range(self.kv):
                for w in (0, 1):
                    self.part[s, layer, h, w].append(host[r:r + n, w, h])
            r += n

    def step(self, seqs, counts, size=1.0, rows=None, layer=None):
        self.extend(seqs, counts)
        batch = self.plan(seqs, counts)
        for l in range(self.layers) if layer is None else [layer]:
            self.append(batch, l, seqs, counts, self.rows(sum(counts), size) if rows is None else rows)
        return batch

    def device_part(self, s, layer, h, which):
        """codes [len, D] and exponents of one sequence, layer and head, from the device's bytes"""
        n, D, N = self.len[s], self.D, self.N
        blocks = -(-n // N)
        g = self.pool.cpu().numpy()[self.pages[s][:blocks, layer, h]][:, :2 * N * D].reshape(blocks, N // 8, 2, 8 * D)
        k = g[:, :, 0].reshape(blocks * N, D)
        v = g[:, :, 1].reshape(blocks, N // 8, D, 8).transpose(0, 1, 3, 2).reshape(blocks * N, D)
        return (k, v)[which][:n], self.exps.cpu().numpy()[s, :blocks, layer, h, which].tolist()

    def check_contents(self):
        torch.cuda.synchronize()
        for (s, l, h, w), part in self.part.items():
            codes, exps = self.device_part(s, l, h, w)
            assert exps == part.exps, (s, l, h, w, exps, part.exps)
            assert np.array_equal(codes, part.codes), (s, l, h, w, int((codes != part.codes).sum()))

    def attend(self, batch, layer, seqs, counts, causal=True, size=1.0, scale=None, weights=None, pad=0, stream=None, q=None):
        """runs the call and holds it to the oracle; returns out"""
        heads, D = self.kv * self.G, self.D
        T = sum(counts)
        scale = D ** -0.5 if scale is None else scale
        width = heads * D + pad
        if q is None:
            q = (torch.from_numpy(self.rng.standard_normal((max(T, 1), width)) * size)).to(self.dtype).cuda()
        out = torch.full((max(T, 1), width), 123.0, dtype=self.dtype, device="cuda")
        torch.cuda.synchronize()
        slora.kv8_attend(batch, layer, q.data_ptr(), width, out.data_ptr(), width, scale, causal, None if weights is None else [t.data_ptr() for t in weights], stream)
        torch.cuda.synchronize()
        self.check_attention(out, q, layer, seqs, counts, causal, scale)
        return out, q

    def check_attention(self, out, q, layer, seqs, counts, causal, scale):
        heads, D = self.kv * self.G, self.D
        host, got = q.double().cpu().numpy(), out.double().cpu().numpy()
        self.drawn = {}
        r0 = 0
        for s, n in zip(seqs, counts):
            size = self.len[s]
            visible = [size - n + 1 + r if causal else size for r in range(n)]
            for h in range(self.kv):
                k, v = (self.part[s, layer, h, w].values() for w in (0, 1))
                total, slack = np.zeros(size), np.zeros(size)
                for m in range(self.G):
                    cols = slice((h * self.G + m) * D, (h * self.G + m + 1) * D)
                    ref, p, bound, p_rel = np_kv8.attention(host[r0:r0 + n, cols], k, v, scale, visible)
                    mine = got[r0:r0 + n, cols]
                    assert np.array_equal(np.isnan(mine), np.isnan(ref)), (s, h, m)
                    ok = ~np.isnan(ref)
                    half = np.abs(ref) * 2.0 ** (-11 if self.dtype == torch.float16 else -8) + 2.0 ** -24
                    err = np.abs(mine - ref)
                    assert (err[ok] <= (bound + half)[ok]).all(), (s, h, m, float((err - bound - half)[ok].max()), float(err[ok].max()))
                    total += p.sum(axis=0)
                    slack += (p * p_rel[:, None]).sum(axis=0) + 1e-37
                self.drawn[s, h] = total, slack
            r0 += n
        if out.shape[1] > heads * D:
            assert (out[:, heads * D:] == 123.0).all()

    def weight_arrays(self):
        shape = (self.max_seqs, self.kv, self.max_tokens)
        w = torch.from_numpy(self.rng.random(shape).astype(np.float32)).cuda()
        return w, torch.full_like(w, -1.0), torch.full(shape, -1, dtype=torch.int32, device="cuda")

    def close(self):
        torch.cuda.synchronize()
        for b in self.batches:
            slora.kv8_batch_destroy(b)
        slora.kv8_destroy(self.cache)
        slora.pool_destroy(self.lib_pool)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
