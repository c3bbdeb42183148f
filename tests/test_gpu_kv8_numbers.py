"""Numbers that attention over the 8-bit cache may meet and that a mean over tokens hides: infinities and NaN in parts of a cache, weights beside
them, ranges far apart.  Against the oracle in 64 bits with its bounds; NaN has to be where the definition has it, and nowhere else."""
import numpy as np
import pytest
import torch

from kv8_util import Twin
from oracle import np_kv8
from paper_2311_03285_amd import slora

pytestmark = pytest.mark.gpu

# new tokens of a sequence, heads that share one of the cache: weights from kept scores, weights from K again behind either form of attention
PATHS = [(5, 2), (12, 2), (40, 2)]


def check_weights(t, seqs, counts, before, after):
    """after = before + what the oracle says the tokens drew, NaN where that is NaN"""
    for s, n in zip(seqs, counts):
        size = t.len[s]
        for h in range(t.kv):
            total, slack = t.drawn[s, h]
            ref = total.copy()
            old = max(size - n, 0)
            ref[:old] += before[s, h, :old]
            got = after[s, h, :size]
            assert np.array_equal(np.isnan(got), np.isnan(ref)), (s, h, np.nonzero(np.isnan(got) != np.isnan(ref))[0])
            ok = ~np.isnan(ref)
            # a row of NaN has no bound: that of the others, 2^-22 * (D + 8) * sum |k| |q| / sqrt(D) and little besides, is under 2^-13 for normal values and D = 32
            slack = np.where(np.isnan(slack), 2.0 ** -13 * ref, slack)
            assert (np.abs(got - ref)[ok] <= (slack + np.abs(ref) * 2.0 ** -22)[ok]).all(), (s, h)
            assert np.array_equal(after[s, h, size:], np.full(t.max_tokens - size, -1.0, np.float32))


def attend_with_weights(t, batch, seqs, counts, **kw):
    w_in, w_out, pos = t.weight_arrays()
    out, q = t.attend(batch, 0, seqs, counts, weights=(w_in, w_out, pos), **kw)
    check_weights(t, seqs, counts, w_in.cpu().numpy(), w_out.cpu().numpy())
    return out, q


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,G", PATHS)
def test_a_bad_v_spoils_outputs_and_no_weight(n, G, dtype):
    """the weights are of scores alone, whatever V holds"""
    with Twin(512, 32, 2, G, dtype, max_seqs=2, max_tokens=200) as t:
        rows = t.rows(100 + 33)
        rows[20, 1, 0, 3] = float("inf")  # sequence 0, head 0, an old token
        t.step([0, 1], [100, 33], rows=rows)
        new = t.rows(2 * n)
        new[n + n // 2, 1, 1, 9] = float("nan")  # sequence 1, head 1, a new token: earlier rows that do not see its block stay numbers
        batch = t.step([0, 1], [n, n], rows=new)
        out, _ = attend_with_weights(t, batch, [0, 1], [n, n])
        nan = torch.isnan(out)
        assert nan[:n, :G * 32].all() and not nan[:n, G * 32:].any() and not nan[n:, :G * 32].any() and nan[2 * n - 1, G * 32:].all()


def test_a_bad_query_spoils_no_weight_of_a_token_that_it_does_not_see():
    for n, G in PATHS:
        with Twin(512, 32, 1, G, max_seqs=1, max_tokens=200) as t:
            t.step([0], [30])
            batch = t.step([0], [n])
            q = torch.from_numpy(t.rng.standard_normal((n, G * 32))).to(t.dtype).cuda()
            q[1, 32 * (G - 1) + 4] = float("nan")  # the second row, its last head
            attend_with_weights(t, batch, [0], [n], q=q)
            assert np.isnan(t.drawn[0, 0][0][:32]).all() and np.isfinite(t.drawn[0, 0][0][32:]).all()


@pytest.mark.parametrize("n", [4, 25, 60])
def test_rows_that_see_nothing_draw_nothing(n):
    """more rows than tokens, with scores far beyond the exponential's range"""
    with Twin(512, 32, 2, 2, max_seqs=2, max_tokens=100) as t:
        t.step([0, 1], [3, 20])
        batch = t.plan([0, 1], [n, n])
        attend_with_weights(t, batch, [0, 1], [n, n], size=100.0)


@pytest.mark.parametrize("large,small", [(70, None), (100, None), (75, -50), (115, -30)])
@pytest.mark.parametrize("old,n,G", [(60, 1, 2), (60, 5, 2), (60, 12, 2), (60, 40, 2), (3000, 1, 1), (3000, 40, 2)])
def test_v_of_blocks_far_apart(large, small, old, n, G):
    """blocks of V of 2^large beside blocks of zeros or of 2^small: tokens of either have their share in the scores' sum"""
    with Twin(512, 64, 1, G, "bf16", max_seqs=1, max_tokens=3100) as t:  # blocks of 8
        rows = t.rows(old)
        rows[:, 1] *= 0.0 if small is None else 2.0 ** small
        some = torch.arange(old, device="cuda") // 8 % 3 == 1
        if old > 100:
            some &= torch.arange(old, device="cuda") < 500  # parts that have none
        rows[some, 1] = t.rows(int(some.sum()))[:, 1] * 2.0 ** large
        t.step([0], [old], rows=rows)
        new = t.rows(n)
        new[:, 1] *= 0.0 if small is None else 2.0 ** small
        batch = t.step([0], [n], rows=new)
        attend_with_weights(t, batch, [0], [n])
        if n == 1:
            t.attend(batch, 0, [0], [n], size=6.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,bits,size", [(1, 24.25, 6000), (1, 28.25, 120), (40, 20.25, 6000), (40, 26.25, 6000)])
def test_many_small_probabilities_beside_a_large_one(n, bits, size, dtype):
    """A token of great score whose V is in one element, others of 2^-bits of its probability whose V is in another: slora.h promises 11 bits of a
    probability down to 2^-21 of the largest, and multiples of 2^-31 of that below"""
    D, large = 64, 1024.0
    with Twin(512, D, 1, 1, dtype, max_seqs=1, max_tokens=size + n) as t:
        rows = torch.zeros((size + n, 2, 1, D), dtype=t.dtype, device="cuda")
        rows[0, 0, 0, 0] = 1.0
        rows[0, 1, 0, 0] = large
        rows[1:, 1, 0, 1] = large
        t.step([0], [size], rows=rows[:size].contiguous())
        batch = t.step([0], [n], rows=rows[size:].contiguous())
        q = torch.zeros((n, D), dtype=t.dtype, device="cuda")
        q[:, 0] = bits
        out, _ = t.attend(batch, 0, [0], [n], q=q, scale=float(np.log(2.0)))
        got = out[:, 1].double().cpu().numpy()
        tokens = size + np.arange(n)  # of the small ones that each row sees
        total = 1.0 + tokens * 2.0 ** -bits
        ref = large * tokens * 2.0 ** -bits / total
        # each rounded to 11 bits or to a multiple of 2^-31; q times log2 e and the exponential in fp32; one rounding of the output
        each = max(2.0 ** -11 * 2.0 ** -bits, 2.0 ** -32) + 2.0 ** -bits * bits * 2.0 ** -20
        bound = large * tokens * each / total + np.abs(ref) * (2.0 ** -11 if dtype == "f16" else 2.0 ** -8) + 2.0 ** -24
        assert (np.abs(got - ref) <= bound).all(), (got[0], ref[0], bound[0])


@pytest.mark.parametrize("size,n,G", [(120, 1, 1), (5000, 1, 1), (700, 4, 8)])
def test_probabilities_of_single_tokens_keep_22_bits(size, n, G):
    """V of opposite signs for the two halves of the tokens, whose probabilities differ in bits that binary16 does not have: what is left of the sum is the difference"""
    D = 64
    with Twin(512, D, 1, G, "f16", max_seqs=1, max_tokens=size + n) as t:
        rows = torch.zeros((size + n, 2, 1, D), dtype=t.dtype, device="cuda")
        k = torch.from_numpy(t.rng.integers(-100, 101, (size + n) // 2)).to(t.dtype).cuda() / 64  # codes
        rows[0:2 * len(k):2, 0, 0, 0] = k
        rows[1:2 * len(k):2, 0, 0, 0] = k  # pairs of equal scores but for element 1
        rows[1:2 * len(k):2, 0, 0, 1] = 1.0
        rows[0::2, 1, 0, 0], rows[1::2, 1, 0, 0] = 1.0, -1.0
        t.step([0], [size], rows=rows[:size].contiguous())
        batch = t.step([0], [n], rows=rows[size:].contiguous())
        q = torch.zeros((n, G * D), dtype=t.dtype, device="cuda")
        q[:, 0::D] = 1.0
        q[:, 1::D] = 2.0 ** -13  # the second of a pair has 1 + 2^-13 log 2 of the first's probability
        out, _ = t.attend(batch, 0, [0], [n], q=q, scale=float(np.log(2.0)))
        got = out.double().cpu().numpy().reshape(n, G, D)[:, :, 0]
        score = rows[:, 0, 0, :2].double().cpu().numpy() @ [1.0, 2.0 ** -13]
        sign = rows[:, 1, 0, 0].double().cpu().numpy()
        for r in range(n):
            seen = size + r + 1
            p = np.exp2(score[:seen])
            p /= p.sum()
            ref = p @ sign[:seen]
            # 2^-22 of each p; an fp32 argument of the exponential (scores below 2, log2 e in three factors) and its result, that sum's and the other's rounding: 2^-20 of each p is
            # more than all; then one rounding of the output
            assert (np.abs(got[r] - ref) <= 2.0 ** -20 + np.abs(ref) * 2.0 ** -11 + 2.0 ** -24).all(), (got[r], ref)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("old,n,G", [(20, 1, 2), (1500, 1, 2), (20, 40, 2), (1500, 40, 2)])
def test_an_infinite_query_gives_nan_and_not_zero(old, n, G, sign, dtype):
    """all scores of a row that sees tokens are the same infinity: there is no softmax, and 0 is for rows that see none"""
    with Twin(512, 32, 1, G, dtype, max_seqs=1, max_tokens=1600) as t:
        rows = t.rows(old + n)
        rows[:, 0, :, 5] = 1.0
        t.step([0], [old], rows=rows[:old].contiguous())
        batch = t.step([0], [n], rows=rows[old:].contiguous())
        q = torch.from_numpy(t.rng.standard_normal((n, G * 32))).to(t.dtype).cuda()
        q[n // 2, 32 + 5] = sign * float("inf")
        out, _ = attend_with_weights(t, batch, [0], [n], q=q)
        nan = torch.isnan(out)
        assert nan[n // 2, 32:].all() and int(nan.sum()) == 32


@pytest.mark.parametrize("n", [1, 12, 40])
@pytest.mark.parametrize("power", [-120, -110, 114, 118])
def test_queries_at_the_ends_of_bfloat16(power, n):
    """what the scale makes ordinary scores of"""
    with Twin(512, 64, 1, 2, "bf16", max_seqs=2, max_tokens=120) as t:
        t.step([0, 1], [60, 9])
        batch = t.step([0, 1], [n, n])
        attend_with_weights(t, batch, [0, 1], [n, n], size=2.0 ** power, scale=2.0 ** (-3 - power))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 12, 40])
@pytest.mark.parametrize("scale", [-0.125, 0.0, -3.0])
def test_scales_that_are_not_positive(n, scale, dtype):
    with Twin(512, 64, 2, 2, dtype, max_seqs=2, max_tokens=300) as t:
        t.step([0, 1], [200, 9])
        batch = t.step([0, 1], [n, n])
        attend_with_weights(t, batch, [0, 1], [n, n], scale=scale)
