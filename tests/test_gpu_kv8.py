"""GPU parity of the 8-bit KV cache: codes and exponents bit for bit, attention within a bound that is derived per element
(np_kv8.attention: probabilities rounded to 11 bits, fp32 sums, one rounding to the 16-bit type), eviction exactly."""
import numpy as np
import pytest
import torch

from kv8_util import Twin
from oracle import np_kv8
from paper_2311_03285_amd import slora

pytestmark = pytest.mark.gpu


# ---- append ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,H", [(32, 256), (64, 1000), (96, 1544), (128, 4096), (192, 1536), (256, 2056)])
def test_append_in_steps(D, H, dtype):
    """prompts, then single tokens and small runs that begin, fill and cross blocks; later tokens are larger, so blocks are shifted"""
    with Twin(H, D, kv=3, G=1, dtype=dtype, layers=2, max_tokens=400) as t:
        t.step([0, 2, 3], [1, 61, 130])
        for size in (0.1, 1.0, 3.0, 40.0, 0.0):
            t.step([0, 1, 2, 3], [1, 3, 9, 1], size)
            t.step([3, 0], [t.N, 1], size)
        t.check_contents()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append_of_extreme_values(dtype):
    """largest and smallest numbers, halfway cases, powers of two beside 127 times a power of two, zeros"""
    with Twin(512, 32, kv=1, G=1, dtype=dtype, max_tokens=200) as t:
        for pattern in range(6):
            rows = t.rows(7)
            big = 6e4 if dtype == "f16" else 3e38
            fill = [[0.0], [127.0, 126.5, 63.5, 0.5, 1.5, -0.5, 2.5, -127.0], [127.5, 127.0, 128.0, 64.25], [big, -big, 1.0, 1e-7],
                    [6e-8, -6e-8, 0.0], [2.0 ** -60, 2.0 ** -50 if dtype == "bf16" else 2.0 ** -24]][pattern]
            flat = rows.view(-1)
            flat.copy_(torch.tensor(fill, dtype=torch.float64).repeat(-(-flat.numel() // len(fill)))[:flat.numel()].to(t.dtype))
            t.step([pattern % 4], [7], rows=rows)
            t.step([pattern % 4], [2], size=1.0)
        t.check_contents()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_bad_value_spoils_its_block_and_no_other(bad):
    with Twin(512, 32, kv=2, G=2, max_tokens=200) as t:
        t.step([0, 1], [40, 40])
        rows = t.rows(2)
        rows[0, 1, 1, 5] = bad  # V of sequence 0, head 1
        t.step([0, 1], [1, 1], rows=rows)
        batch = t.step([0, 1], [1, 1])
        t.check_contents()
        assert t.part[0, 0, 1, 1].exps[40 // t.N] == np_kv8.POISON
        out, _ = t.attend(batch, 0, [0, 1], [1, 1])
        assert torch.isnan(out[0, 2 * 32:]).all() and not torch.isnan(out[0, :2 * 32]).any() and not torch.isnan(out[1]).any()


# ---- attention ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("kv,G", [(2, 1), (1, 5), (2, 8), (1, 17)])
def test_single_tokens(D, kv, G, dtype):
    """lengths from one, about the ends of granules, chunks of 32 and blocks"""
    with Twin(8 * D + 8 * (D // 8) * 3, D, kv, G, dtype, max_seqs=9, max_tokens=300) as t:
        lens = [1, 2, 7, 8, 9, 31, 33, 129, 290]
        t.step(list(range(9)), [n - 1 for n in lens])
        batch = t.step(list(range(9)), [1] * 9)
        t.attend(batch, 0, list(range(9)), [1] * 9, pad=8)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,kv,G", [(64, 2, 1), (128, 2, 3), (128, 1, 8), (96, 2, 4), (256, 1, 2), (32, 1, 16)])
def test_prompts_and_chunks(D, kv, G, causal, dtype):
    """prompts on an empty cache and behind history, drafted tokens, single tokens, in one call"""
    with Twin(16 * D, D, kv, G, dtype, max_seqs=6, max_tokens=420) as t:
        seqs, counts = [5, 0, 3, 1, 2], [150, 1, 33, 5, 64]
        t.step([0, 1, 2, 4], [200, 37, 300, 9])
        batch = t.step(seqs, counts)
        t.attend(batch, 0, seqs, counts, causal)


@pytest.mark.parametrize("rows", [1, 2, 40])
def test_long_sequences_are_split_and_joined(rows):
    with Twin(1024, 64, 2, 2, "bf16", max_seqs=2, max_tokens=20100) as t:
        t.step([1], [20000 - 17])
        t.step([0], [300])
        batch = t.step([0, 1], [rows, rows])
        t.attend(batch, 0, [0, 1], [rows, rows], size=3.0)


def test_rows_that_see_nothing_are_zero():
    with Twin(512, 64, 2, 2, max_seqs=3, max_tokens=100) as t:
        t.step([1, 2], [3, 50])
        batch = t.plan([0, 1, 2], [4, 10, 2])  # more rows than tokens: attention over what is there
        out, _ = t.attend(batch, 0, [0, 1, 2], [4, 10, 2])
        assert (out[:4 + 7] == 0).all() and (out[11:] != 0).any(dim=1).all()
        out, _ = t.attend(batch, 0, [0, 1, 2], [4, 10, 2], causal=False)
        assert (out[:4] == 0).all()


def test_units_far_apart():
    """V of blocks from 2^-40 to 2^40 times each other, K in large and small units, and large scores"""
    with Twin(512, 64, 1, 2, "bf16", max_seqs=4, max_tokens=100) as t:  # blocks of 8
        for k, size in enumerate([1.0, 2.0 ** -40, 2.0 ** 40, 2.0 ** -20, 1.0, 2.0 ** 10]):
            rows = t.rows(16)
            rows[:, 1] *= size
            rows[8:, 1] *= 2.0 ** -7
            rows[:, 0] *= [1.0, 4.0, 0.25][k % 3]
            t.step([0, 1], [8, 8], rows=rows)
        batch = t.plan([0, 1], [1, 1])
        t.attend(batch, 0, [0, 1], [1, 1])
        t.attend(batch, 0, [0, 1], [1, 1], size=6.0)


@pytest.mark.parametrize("size", [2.0 ** -30, 2.0 ** -8, 1.0, 2.0 ** 40])
def test_queries_of_any_size_in_bfloat16(size):
    with Twin(512, 64, 1, 2, "bf16", max_seqs=2, max_tokens=100) as t:
        t.step([0, 1], [60, 9])
        batch = t.step([0, 1], [3, 1])
        t.attend(batch, 0, [0, 1], [3, 1], size=size, scale=1.0 / (8 * size))


def test_layers_have_their_own_pages():
    with Twin(512, 32, 2, 2, layers=3, max_seqs=2, max_tokens=100) as t:
        t.step([0, 1], [33, 70])
        batch = t.step([0, 1], [1, 4])
        for layer in (2, 0, 1):
            t.attend(batch, layer, [0, 1], [1, 4])
        t.check_contents()


def test_pages_beyond_four_gigabytes():
    """byte offsets of pages need 33 bits"""
    n_pages = 300000  # of 16 KiB
    fill = lambda n, width: torch.empty((n, width), dtype=torch.int8, device="cuda")
    with Twin(8192, 128, 1, 2, "f16", max_seqs=2, max_tokens=700, n_pages=n_pages, fill=fill) as t:
        t.free = list(range(n_pages - 100, n_pages))
        t.step([0, 1], [600, 64])
        batch = t.step([0, 1], [1, 2])
        assert int(t.pages[0].min()) * 16384 > 1 << 32
        t.device_pool = t.pool
        small = t.pool[n_pages - 100:]
        for s in (0, 1):  # (check_contents would copy the whole pool)
            pages = t.pages[s][:, 0, 0] - (n_pages - 100)
            k = small[torch.from_numpy(pages.astype(np.int64)).cuda()].cpu().numpy().reshape(len(pages), 8, 2, 1024)[:, :, 0].reshape(-1, 128)
            assert np.array_equal(k[:t.len[s]], t.part[s, 0, 0, 0].codes)
        t.attend(batch, 0, [0, 1], [1, 2])


def test_other_streams_and_the_order_of_a_batch():
    with Twin(512, 64, 2, 2, max_seqs=2, max_tokens=400) as t:
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        t.step([0, 1], [200, 100])
        torch.cuda.synchronize()
        t.extend([0, 1], [1, 1])
        batch = t.plan([0, 1], [1, 1])
        rows = t.rows(2)
        torch.cuda.synchronize()
        width = t.kv * t.D
        slora.kv8_append(batch, 0, rows.data_ptr(), 2 * width, rows.data_ptr() + 2 * width, 2 * width, a)
        host = rows.double().cpu().numpy()
        for s in (0, 1):
            for h in range(t.kv):
                for w in (0, 1):
                    t.part[s, 0, h, w].append(host[s:s + 1, w, h])
        t.attend(batch, 0, [0, 1], [1, 1], stream=b)


def test_a_graph_replays_a_step():
    """append and attend of a layer captured once, replayed with other inputs in the same buffers"""
    with Twin(512, 64, 2, 4, "bf16", max_seqs=2, max_tokens=900) as t:
        t.step([0, 1], [800, 9])
        t.extend([0, 1], [1, 1])
        batch = t.plan([0, 1], [1, 1])
        width, heads = t.kv * t.D, t.kv * t.G
        rows, q = t.rows(2), torch.zeros((2, heads * t.D), dtype=t.dtype, device="cuda")
        out = torch.zeros_like(q)
        w = t.weight_arrays()

        def call(stream):
            slora.kv8_append(batch, 0, rows.data_ptr(), 2 * width, rows.data_ptr() + 2 * width, 2 * width, stream)
            slora.kv8_attend(batch, 0, q.data_ptr(), heads * t.D, out.data_ptr(), heads * t.D, 0.125, True, [x.data_ptr() for x in w], stream)

        stream = torch.cuda.Stream()
        call(stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(torch.cuda.current_stream())
        for _ in range(3):
            q.copy_(torch.from_numpy(t.rng.standard_normal(q.shape)))
            graph.replay()
            torch.cuda.synchronize()
            mine, drawn = out.clone(), w[1].clone()
            out.zero_()
            w[1].fill_(-1.0)
            call(stream)
            torch.cuda.synchronize()
            assert torch.equal(mine, out) and torch.equal(drawn, w[1])


# ---- weights ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,kv,G,counts", [(64, 2, 1, [1, 1, 1]), (128, 2, 8, [1, 1, 1]), (96, 1, 3, [40, 1, 7]), (256, 2, 2, [130, 3, 1]), (32, 1, 20, [1, 2, 30])])
def test_weights_that_tokens_draw(D, kv, G, counts, dtype):
    with Twin(16 * D, D, kv, G, dtype, max_seqs=4, max_tokens=500) as t:
        seqs = [2, 0, 3]
        t.step(seqs, [300, 5, 77])
        batch = t.step(seqs, counts)
        w_in, w_out, pos = t.weight_arrays()
        t.attend(batch, 0, seqs, counts, weights=(w_in, w_out, pos))
        first, before = w_out.cpu().numpy(), w_in.cpu().numpy()
        for s, n in zip(seqs, counts):
            size = t.len[s]
            for h in range(kv):
                total, slack = t.drawn[s, h]
                ref = total.copy()
                ref[:size - n] += before[s, h, :size - n]
                got = first[s, h]
                assert (np.abs(got[:size] - ref) <= slack + np.abs(ref) * 2.0 ** -22).all()
                assert (got[size:] == -1).all()
                assert np.array_equal(pos[s, h, size - n:size].cpu().numpy(), np.arange(size - n, size))
                assert (pos[s, h, :size - n] == -1).all()
        assert (first[1] == -1).all()
        # in place, and again: the same bits
        t.attend(batch, 0, seqs, counts, weights=(w_in, w_in, pos), q=torch.zeros((sum(counts), kv * G * D), dtype=t.dtype, device="cuda"))
        for s, n in zip(seqs, counts):
            assert not torch.equal(w_in[s, 0, :t.len[s]], torch.from_numpy(before[s, 0, :t.len[s]]).cuda())


# ---- eviction ---------------------------------------------------------------------------------------
def evict_and_check(t, seqs, keep, recent, w, pos, in_place=False, layer=0):
    batch = t.plan(seqs, [0] * len(seqs), keep)
    w_out, pos_out = (w, pos) if in_place else (torch.full_like(w, -1.0), torch.full_like(pos, -1))
    before_w, before_p = w.cpu().numpy().copy(), pos.cpu().numpy().copy()
    slora.kv8_evict(batch, layer, recent, w.data_ptr(), w_out.data_ptr(), pos.data_ptr(), pos_out.data_ptr())
    torch.cuda.synchronize()
    for s, n in zip(seqs, keep):
        n = min(n, t.len[s])
        for h in range(t.kv):
            moves, ww, pp = np_kv8.evict(before_w[s, h, :t.len[s]], before_p[s, h, :t.len[s]], t.seen[s], n, recent)
            assert np.array_equal(w_out[s, h, :n].cpu().numpy(), ww, equal_nan=True), (s, h)
            assert np.array_equal(pos_out[s, h, :n].cpu().numpy(), pp), (s, h)
            if n < t.len[s]:
                for which in (0, 1):
                    t.part[s, layer, h, which].move(moves, n)
            if not in_place:
                assert (w_out[s, h, n:] == -1).all()
    t.truncate(seqs, [min(n, t.len[s]) for s, n in zip(seqs, keep)], evicted=True)
    t.check_contents()
    return w_out, pos_out


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("keep,recent", [([120, 300, 8, 40], 10), ([121, 1, 299, 0], 0), ([64, 63, 65, 300], 64), ([7, 150, 16, 33], 1000)])
@pytest.mark.parametrize("D,H", [(32, 512), (96, 1536), (128, 4096)])
def test_eviction(D, H, keep, recent, in_place):
    with Twin(H, D, 3, 2, max_seqs=4, max_tokens=320) as t:
        for size in (1.0, 0.03, 8.0):
            t.step([0, 1, 2, 3], [100, 90, 99, 13], size)
        w, _, pos = t.weight_arrays()
        w[t.rng.random(w.shape) < 0.3] = 0.5  # many equal weights
        for s in range(4):
            pos[s, :, :t.len[s]] = torch.arange(t.len[s], device="cuda", dtype=torch.int32)
        w2, p2 = evict_and_check(t, [0, 1, 2, 3], keep, recent, w, pos, in_place)
        # the cache goes on: new tokens behind those that stayed
        batch = t.step([0, 1, 2, 3], [1, 12, 1, 1])
        t.attend(batch, 0, [0, 1, 2, 3], [1, 12, 1, 1], weights=(w2, w2, p2))
        assert int(p2[1, 0, t.len[1] - 1]) == t.seen[1] - 1


def test_eviction_by_odd_weights():
    """NaN, infinities, both zeros, negative and subnormal weights, all equal, more recent ones than stay"""
    with Twin(512, 64, 2, 1, max_seqs=4, max_tokens=200) as t:
        t.step([0, 1, 2, 3], [100, 100, 100, 100])
        w, _, pos = t.weight_arrays()
        for s in range(4):
            pos[s, :, :100] = torch.from_numpy(t.rng.permutation(100).astype(np.int32)).cuda()
        odd = torch.tensor([np.nan, -np.inf, np.inf, 0.0, -0.0, -1.0, 1e-42, -1e-42, 3.0, np.nan], dtype=torch.float32, device="cuda")
        w[0, :, :100] = odd.repeat(10)
        w[1] = 0.25
        w[2, :, :100] = torch.cat([odd, -odd]).repeat(5)
        evict_and_check(t, [0, 1, 2, 3], [37, 50, 61, 20], 30, w, pos)


def test_eviction_of_long_sequences_step_by_step():
    """a cache at its budget: one token over it after each step"""
    with Twin(2048, 64, 2, 2, "bf16", max_seqs=2, max_tokens=5000) as t:
        t.step([0, 1], [4500, 700])
        w, _, pos = t.weight_arrays()
        for s in range(2):
            pos[s, :, :t.len[s]] = torch.arange(t.len[s], device="cuda", dtype=torch.int32)
        evict_and_check(t, [0, 1], [401, 401], 50, w, pos, in_place=True)
        for _ in range(3):
            batch = t.step([1, 0], [1, 1])
            t.attend(batch, 0, [1, 0], [1, 1], weights=(w, w, pos))
            evict_and_check(t, [1, 0], [401, 401], 50, w, pos, in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("D,H,dtype", [(32, 512, "f16"), (64, 512, "bf16"), (128, 4096, "f16"), (192, 1536, "f16"), (256, 2048, "bf16")])
def test_eviction_of_a_few_tokens(D, H, dtype, in_place):
    """none to four tokens over the budget, equal weights, tokens that are themselves behind it, blocks in smaller units than what comes"""
    with Twin(H, D, 5, 1, dtype, max_seqs=6, max_tokens=400) as t:
        for size in (0.05, 1.0, 9.0):
            t.step([0, 1, 2, 3, 4, 5], [100, 3, 60, 61, 2, 110], size)
        lens = list(t.len)
        w, _, pos = t.weight_arrays()
        w[t.rng.random(w.shape) < 0.5] = 0.0
        w[2, 1] = 0.0
        w[3, 2, :20], w[3, 2, 5] = float("nan"), -0.0
        w[5, :, lens[5] - 4:] = 0.0  # the last ones go, or stay as recent
        for s in range(6):
            pos[s, :, :lens[s]] = torch.arange(lens[s], device="cuda", dtype=torch.int32)
        keep = [lens[0] - 4, lens[1] - 1, lens[2] - 3, lens[3], lens[4] - 4, lens[5] - 2]
        for recent in (0, 3):
            w, pos = evict_and_check(t, [0, 1, 2, 3, 4, 5], keep, recent, w, pos, in_place)
            t.step([0, 1, 2, 3, 4, 5], [4, 1, 3, 0, 2, 2], 20.0 * (recent + 1))
            for s, n in enumerate([4, 1, 3, 0, 2, 2]):
                w[s, :, t.len[s] - n:t.len[s]] = 0.125 * s
                pos[s, :, t.len[s] - n:t.len[s]] = torch.arange(t.seen[s] - n, t.seen[s], device="cuda", dtype=torch.int32)
        evict_and_check(t, [4, 1], [1, 0], 0, w, pos, in_place)


def test_eviction_of_a_few_tokens_of_many_rows_with_long_ones():
    """512 rows, the longest of which are read four times by one wavefront"""
    with Twin(512, 32, 32, 1, max_seqs=16, max_tokens=2100) as t:
        every, size = list(range(16)), [20 + 3 * s for s in range(15)] + [2049]
        t.step(every, size)
        w, _, pos = t.weight_arrays()
        w[t.rng.random(w.shape) < 0.5] = 0.0
        for s in every:
            pos[s, :, :size[s]] = torch.arange(size[s], device="cuda", dtype=torch.int32)
        evict_and_check(t, every, [size[s] - s % 5 for s in range(15)] + [2045], 15, w, pos)


@pytest.mark.parametrize("size", [4096, 4097, 4160])
def test_eviction_about_the_length_from_which_a_row_has_more_wavefronts(size):
    with Twin(2048, 64, 2, 1, max_seqs=2, max_tokens=4200) as t:
        t.step([0, 1], [size, 70])
        w, _, pos = t.weight_arrays()
        w[t.rng.random(w.shape) < 0.3] = 0.5
        for s in range(2):
            pos[s, :, :t.len[s]] = torch.arange(t.len[s], device="cuda", dtype=torch.int32)
        evict_and_check(t, [0, 1], [size - 100, 64], 50, w, pos)


def test_a_table_entry_that_is_given_another_page():
    """truncate, then grow again on other pages while earlier work may still run"""
    with Twin(512, 64, 1, 2, max_seqs=2, max_tokens=200) as t:
        t.step([0, 1], [60, 60])
        for n in (33, 8, 0):
            t.truncate([0], [n])
            t.free.reverse()
            batch = t.step([0, 1], [40, 1])
            t.attend(batch, 0, [0, 1], [40, 1])
        t.check_contents()
