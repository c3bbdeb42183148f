"""Served layers: base projections in 4 bits or 8, LoRA, the 8-bit KV cache and its eviction in one pool; with 8 bits, norms and a feed-forward block.

    python -m paper_2311_03285_amd.attention_layer [--bits 8 [--wide 16384]]

serves three requests with adapters of different ranks: prompts first, then a token each, until the cache is at its budget and every
further token takes the place of another.  For each step the host extends the sequences and plans the batch once;
per layer the device runs

    q, k, v = x W + (x A) B       slora_w4_matmul_y16 for three matrices, then slora_lora_apply_multi_y16
    cache  <- k, v                slora_kv8_append
    a       = attention(q)        slora_kv8_attend, adding up what every cached token draws
    out     = a W + (a A) B       the same two calls for the fourth projection
    cache  -> budget              slora_kv8_evict

With 8-bit base weights (--bits 8) the layers are whole ones, around a residual stream h:

    x      = norm(h)              slora_norm_apply, in 16 bits for LoRA and in 8 for the products
    q, k, v, cache, a             as above, with slora_w8_matmul_y16
    out    = a W + (a A) B        slora_w8_quantize of a, then the same two calls
    h      = h + out, normalised  slora_norm_apply
    g, u   = x W                  slora_w8_matmul_y16 for two wide matrices
    block  = (silu(g) u) W        slora_w8_quantize of the gated product, slora_w8_matmul_y16
    h      = h + block            slora_norm_apply, which normalises for the next layer

Everything runs on one stream and nothing waits for the host.  (Positions are not encoded here: a model rotates q and k before they go in.)
"""
from __future__ import annotations

import argparse
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import slora

DTYPES = {slora.F16: torch.float16, slora.BF16: torch.bfloat16}


class AttentionLayer:
    """One pool, one cache and the weights of `layers` layers.  All projections map H -> H, as LoRA's do here; heads of H / n_heads elements.
    bits: of the base weights.  With 8, layers have norms, residuals and - if wide > 0 - a feed-forward block of that width."""

    def __init__(self, H: int, n_heads: int, layers: int, pool_pages: int, max_seqs: int, max_tokens: int, budget: int, recent: int, ranks: Dict[int, int],
                 group: int = 128, dtype: int = slora.F16, seed: int = 0, device="cuda", bits: int = 4, wide: int = 0):
        if bits not in (4, 8) or wide < 0 or (wide and bits == 4):
            raise ValueError("bits must be 4 or 8, and a feed-forward block needs 8")
        if bits == 8 and (H > slora.NORM_MAX_WIDTH or wide > slora.W8_MAX_WIDTH):
            raise ValueError(f"norms are of rows up to {slora.NORM_MAX_WIDTH} wide, gated products up to {slora.W8_MAX_WIDTH}")
        self.bits, self.wide, self.lib_dtype = bits, wide, dtype
        self.H, self.n_heads, self.D, self.layers, self.budget, self.recent, self.dtype = H, n_heads, H // n_heads, layers, budget, recent, DTYPES[dtype]
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.pages = torch.empty((pool_pages, H), dtype=self.dtype, device=device)
        self.pool = slora.pool_init(H, pool_pages, dtype, self.pages.data_ptr(), 4 * layers, max(ranks.values()))
        self.exps = torch.empty((max_seqs * slora.kv8_block_count(H, self.D, max_tokens) * layers * n_heads * 2,), dtype=torch.int8, device=device)
        self.cache = slora.kv8_init(self.pool, layers, n_heads, n_heads, self.D, max_seqs, max_tokens, self.exps.data_ptr())
        self.weights = [torch.zeros((max_seqs, n_heads, max_tokens), device=device) for _ in range(layers)]
        self.pos = [torch.zeros((max_seqs, n_heads, max_tokens), dtype=torch.int32, device=device) for _ in range(layers)]
        # Packing and uploads run on torch's stream, behind the operations there that make what they read.
        stream = torch.cuda.current_stream()
        # base weights: codes about 8, a scale per group; slot 4 * layer + (0, 1, 2, 3) is q, k, v, o, for LoRA as well
        self.codes, self.scales, self.packed, self.matrices, self.norms = [], [], [], [], []
        for _ in range(4 * layers if bits == 4 else 0):
            c = (torch.randn((H, H), device=device, generator=g) * 2.6 + 8).round_().clamp_(0, 15).to(torch.uint8)
            s = ((0.5 + torch.rand((H, -(-H // group)), device=device, generator=g)) / (2.6 * H ** 0.5)).to(self.dtype)
            packed = torch.empty(slora.w4_bytes(H, H, group), dtype=torch.uint8, device=device)
            nibbles = (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous()
            self.matrices.append(slora.w4_pack(H, H, group, dtype, nibbles.data_ptr(), s.data_ptr(), None, packed.data_ptr(), stream))
            self.codes.append(c)
            self.scales.append(s)
            self.packed.append(packed)
            torch.cuda.synchronize()  # (nibbles may go)
        if bits == 8:
            self._weights_of_8_bits(g, stream)
        self.group = group
        self.adapters: Dict[int, torch.Tensor] = {}
        for a, r in ranks.items():
            slora.adapter_alloc(self.pool, a, r, 4 * layers)
            w = torch.randn((4 * layers, 2, r, H), device=device, generator=g)
            w[:, 0] /= H ** 0.5
            w[:, 1] /= 4 * r ** 0.5
            self.adapters[a] = w.to(self.dtype)
            slora.adapter_upload(self.pool, a, self.adapters[a].data_ptr(), stream)
        torch.cuda.synchronize()  # (steps may run on another stream)

    def _weights_of_8_bits(self, g, stream) -> None:
        """... as above, and behind them gate, up and down of each layer; a norm before each half of a layer, and one that adds the last block"""
        H, wide, layers, device = self.H, self.wide, self.layers, self.pages.device
        shapes = [(H, H)] * (4 * layers) + ([(wide, H), (wide, H), (H, wide)] * layers if wide else [])
        for outputs, inputs in shapes:
            self.codes.append((torch.randn((outputs, inputs), device=device, generator=g) * 35).round_().clamp_(-127, 127).to(torch.int8))
            self.scales.append((0.5 + torch.rand((outputs,), device=device, generator=g)) / (35 * inputs ** 0.5))
            self.packed.append(torch.empty(slora.w8_bytes(outputs, inputs), dtype=torch.uint8, device=device))
            self.matrices.append(slora.w8_pack(outputs, inputs, self.lib_dtype, self.codes[-1].data_ptr(), self.scales[-1].data_ptr(), self.packed[-1].data_ptr(),
                                               stream))
        self.norm_weights = [(1 + 0.2 * torch.randn((H,), device=device, generator=g)).to(self.dtype) for _ in range((2 if wide else 1) * layers)]
        self.norms = [slora.norm_init(H, self.lib_dtype, pre_weight=w.data_ptr()) for w in self.norm_weights] + [slora.norm_init(H, self.lib_dtype)]

    def step(self, seqs: Sequence[int], tokens: Sequence[int], adapters: Sequence[int], x: torch.Tensor) -> List[torch.Tensor]:
        """x: [sum of tokens, H], new tokens of `seqs` (whose adapters are given); returns every layer's output, each layer reading the one before.
        A step that is refused (an adapter that is not loaded, no pages left) leaves the sequences as they were."""
        if x.shape != (sum(tokens), self.H) or x.dtype != self.dtype or x.device != self.pages.device or not x.is_contiguous():
            raise ValueError(f"x must be [{sum(tokens)}, {self.H}] of {self.dtype} on {self.pages.device}, row after row")
        if not len(seqs) == len(tokens) == len(adapters):
            raise ValueError("as many tokens and adapters as sequences")
        before = slora.kv8_lengths(self.cache, seqs)
        slora.kv8_extend(self.cache, seqs, tokens)
        batch = plan = None
        try:
            lengths = slora.kv8_lengths(self.cache, seqs)
            keep = np.minimum(lengths, self.budget)
            evicts = bool((keep < lengths).any())
            batch = slora.kv8_batch_plan(self.cache, seqs, tokens, keep)
            plan = slora.batch_plan(self.pool, np.repeat(np.asarray(adapters, np.int32), tokens), np.concatenate([[0], np.cumsum(tokens)]))
            outputs = (self._layers if self.bits == 4 else self._whole_layers)(batch, plan, x, evicts)
        except Exception:
            slora.kv8_truncate(self.cache, seqs, before)  # (what is refused is refused before anything is launched)
            raise
        finally:
            if plan is not None:
                slora.plan_destroy(plan)
            if batch is not None:
                slora.kv8_batch_destroy(batch)
        if evicts:
            slora.kv8_truncate(self.cache, seqs, keep, evicted=True)
        return outputs

    def _layers(self, batch, plan, x: torch.Tensor, evicts: bool) -> List[torch.Tensor]:
        H, D, T, stream = self.H, self.D, x.shape[0], torch.cuda.current_stream()
        outputs = []
        for layer in range(self.layers):
            q, k, v, a, out = (torch.empty((T, H), dtype=self.dtype, device=x.device) for _ in range(5))
            slots = [4 * layer + i for i in range(3)]
            ys = [t.data_ptr() for t in (q, k, v)]
            slora.w4_matmul_y16([self.matrices[s] for s in slots], [x.data_ptr()] * 3, T, ys, stream)
            slora.lora_apply_multi_y16(plan, slots, [x.data_ptr()] * 3, ys, stream)
            w, p = self.weights[layer].data_ptr(), self.pos[layer].data_ptr()
            slora.kv8_append(batch, layer, k.data_ptr(), H, v.data_ptr(), H, stream)
            slora.kv8_attend(batch, layer, q.data_ptr(), H, a.data_ptr(), H, D ** -0.5, True, (w, w, p), stream)
            slora.w4_matmul_y16([self.matrices[4 * layer + 3]], [a.data_ptr()], T, [out.data_ptr()], stream)
            slora.lora_apply_multi_y16(plan, [4 * layer + 3], [a.data_ptr()], [out.data_ptr()], stream)
            if evicts:
                slora.kv8_evict(batch, layer, self.recent, w, w, p, p, stream)
            outputs.append(out)
            x = out
        return outputs

    def _whole_layers(self, batch, plan, h: torch.Tensor, evicts: bool) -> List[torch.Tensor]:
        H, D, wide, T, stream = self.H, self.D, self.wide, h.shape[0], torch.cuda.current_stream()
        rows = lambda n: torch.empty((T, n), dtype=self.dtype, device=h.device)
        scales, codes = torch.empty((T,), device=h.device), torch.empty((T, -(-max(H, wide) // 16) * 16), dtype=torch.int8, device=h.device)
        norms, block, outputs = iter(self.norms), None, []

        def norm(h: torch.Tensor, block: Optional[torch.Tensor], x: Optional[torch.Tensor], more: bool = True) -> torch.Tensor:
            """h + block; that normalised, in 16 bits if x is given, in 8 if there is more to come"""
            out = h if block is None else rows(H)
            added = {} if block is None else dict(block=block.data_ptr(), block_stride=block.stride(0), h_out=out.data_ptr(), h_out_stride=H)
            if x is not None:
                added.update(x=x.data_ptr(), x_stride=H)
            if more:
                added.update(codes=codes.data_ptr(), codes_stride=codes.stride(0), scales=scales.data_ptr())
            slora.norm_apply(next(norms), T, h.data_ptr(), H, **added, stream=stream)
            return out

        def product(first: int, ys: List[torch.Tensor]) -> None:
            n = len(ys)
            slora.w8_matmul_y16(self.matrices[first:first + n], [codes.data_ptr()] * n, [codes.stride(0)] * n, [scales.data_ptr()] * n, T, [y.data_ptr() for y in ys],
                                [y.stride(0) for y in ys], stream)

        def quantize(x: torch.Tensor, width: int, gate: Optional[torch.Tensor] = None) -> None:
            slora.w8_quantize(T, width, self.lib_dtype, slora.ACT_NONE if gate is None else slora.ACT_SILU, x.data_ptr(), x.stride(0),
                              None if gate is None else gate.data_ptr(), 0 if gate is None else gate.stride(0), codes=codes.data_ptr(), codes_stride=codes.stride(0),
                              scales=scales.data_ptr(), stream=stream)

        for layer in range(self.layers):
            x, q, k, v, a, out = (rows(H) for _ in range(6))
            slots = [4 * layer + i for i in range(3)]
            ys = [t.data_ptr() for t in (q, k, v)]
            h = norm(h, block, x)
            if layer > 0:
                outputs.append(h)
            product(4 * layer, [q, k, v])
            slora.lora_apply_multi_y16(plan, slots, [x.data_ptr()] * 3, ys, stream)
            w, p = self.weights[layer].data_ptr(), self.pos[layer].data_ptr()
            slora.kv8_append(batch, layer, k.data_ptr(), H, v.data_ptr(), H, stream)
            slora.kv8_attend(batch, layer, q.data_ptr(), H, a.data_ptr(), H, D ** -0.5, True, (w, w, p), stream)
            quantize(a, H)
            product(4 * layer + 3, [out])
            slora.lora_apply_multi_y16(plan, [4 * layer + 3], [a.data_ptr()], [out.data_ptr()], stream)
            if evicts:
                slora.kv8_evict(batch, layer, self.recent, w, w, p, p, stream)
            block = out
            if wide:
                # (rows of the wide products begin 16 bytes apart, whatever their width)
                gate, up, block = rows(-(-wide // 8) * 8), rows(-(-wide // 8) * 8), rows(H)
                first = 4 * self.layers + 3 * layer
                h = norm(h, out, None)
                product(first, [gate, up])
                quantize(up, wide, gate)
                product(first + 2, [block])
        return outputs + [norm(h, block, None, more=False)]

    def finish(self, seqs: Sequence[int]) -> None:
        """Requests that are done: their pages are free for other requests and for adapters."""
        slora.kv8_truncate(self.cache, seqs, [0] * len(seqs))

    def close(self) -> None:
        torch.cuda.synchronize()
        for m in self.matrices:
            (slora.w4_destroy if self.bits == 4 else slora.w8_destroy)(m)
        for n in self.norms:
            slora.norm_destroy(n)
        slora.kv8_destroy(self.cache)
        slora.pool_destroy(self.pool)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--bits", type=int, default=4, choices=(4, 8), help="of the base weights; with 8, whole layers")
    parser.add_argument("--wide", type=int, default=None, help="width of the feed-forward block of whole layers (default 16384; 0: none)")
    args = parser.parse_args()
    if args.wide is not None and args.bits == 4:
        parser.error("--wide needs --bits 8")
    wide = 0 if args.bits == 4 else 16384 if args.wide is None else args.wide
    with AttentionLayer(H=4096, n_heads=32, layers=2, pool_pages=20000, max_seqs=8, max_tokens=700, budget=512, recent=64, ranks={0: 8, 1: 16, 2: 64}, bits=args.bits,
                        wide=wide) as m:
        x = torch.randn((400 + 510 + 37, 4096), device="cuda").to(m.dtype)
        m.step([0, 1, 2], [400, 510, 37], [0, 1, 2], x)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for i in range(24):
            if i == 4:
                start.record()
            out = m.step([0, 1, 2], [1, 1, 1], [0, 1, 2], torch.randn((3, 4096), device="cuda").to(m.dtype))
        end.record()
        torch.cuda.synchronize()
        lengths, pages = slora.kv8_lengths(m.cache, [0, 1, 2]).tolist(), slora.kv8_info(m.cache)["pages"]
        print(f"lengths {lengths} of at most {m.budget}, {pages} pages of cache, {slora.pool_free_pages(m.pool)} free; "
              f"{start.elapsed_time(end) / 20 * 1e3:.0f} us a step of {m.layers} layers; output rms {out[-1].float().pow(2).mean().sqrt():.3f}")
        m.finish([0, 1, 2])


if __name__ == "__main__":
    main()
