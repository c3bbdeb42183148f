// gfx950 kernels of the 8-bit KV cache: append, attention, the weights that cached tokens draw, eviction.
//
// Layout (see slora.h): a page holds a block of N tokens of one head, in granules of eight - 8 * D bytes of
// K as [token][element], 8 * D bytes of V as [element][token].  A code c stands for c * 2^e, e by block.
// All byte offsets into the pool are 64-bit.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "kv8.hpp"

namespace slora {

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float across_16(float v) { return __shfl_xor(v, 16, kWave); }
__device__ __forceinline__ float across_32(float v) { return __shfl_xor(v, 32, kWave); }

// n / (granules per block) by div = ceil(2^32 / d): exact while n * d < 2^32, and n < 2^24 granules, d <= 128; 0 stands for d = 1
__device__ __forceinline__ uint32_t kv_div(uint32_t n, uint32_t div) { return div ? __umulhi(n, div) : n; }

__device__ __forceinline__ int64_t table_entry(const KvShape &s, int seq, int block, int head)
{
    return (((int64_t)seq * s.max_blocks + block) * s.n_layers + s.layer) * s.n_kv + head;
}

// 2^e of a block: NaN for one that holds an infinity or NaN
__device__ __forceinline__ float unit_of(int e) { return e == kKvPoison ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(e + 127) << 23); }

// least e >= kKvLowest with amax <= 127 * 2^e = 1.984375 * 2^(e + 6); amax >= 0
__device__ __forceinline__ int exponent_of(float amax)
{
    const int32_t bits = __float_as_int(amax);
    if (bits >= 0x7f800000) return kKvPoison;
    return max(((bits - 0x7e0001) >> 23) - 132, kKvLowest);
}

// code of `v` in units of 2^e (|v| <= 127 * 2^e): the product is exact, so this is the only rounding
__device__ __forceinline__ int code_of(float v, float inverse) { return (int)__builtin_rintf(v * inverse); }

// 2^-e of a block without infinities (e <= 122: the bits of a normal number)
__device__ __forceinline__ float inverse_of(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }

// the four codes in `u` in units 2^shift times larger (shift >= 0): each rounded to nearest, ties to even
__device__ __forceinline__ uint32_t shift_codes(uint32_t u, float factor)
{
    uint32_t r = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) r |= ((uint32_t)(int)__builtin_rintf((float)(int8_t)(u >> (8 * k)) * factor) & 0xffu) << (8 * k);
    return r;
}
__device__ __forceinline__ float shift_factor(int from, int to) // both exponents of a block; 0 where it becomes poisoned
{
    return to == kKvPoison || to - from > 100 ? 0.0f : __uint_as_float((uint32_t)(127 - (to - from)) << 23);
}

// ---------------------------------------------------------------------------------------
// page table
// ---------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void kv_table_kernel(int32_t *__restrict__ table, const int32_t *__restrict__ columns, const int32_t *__restrict__ pages, int per)
{
    const int64_t to = (int64_t)columns[blockIdx.x] * per, from = (int64_t)blockIdx.x * per;
    for (int i = threadIdx.x; i < per; i += blockDim.x) table[to + i] = pages[from + i];
}

// ---------------------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------------------
// A workgroup = the new tokens of one block and head; wavefront 0 writes K, wavefront 1 V.  Each reads its rows twice (the second time
// they are in the caches): once for the largest value, once to round them.  K: 16 bytes of a row a lane.  V, which is
// stored transposed: a lane has two elements of the eight tokens of a granule, reads them as 4 bytes of eight rows and writes
// 16 bytes; what the granule held before stays, in new units if the exponent has grown.
// Bound: latency (item, page, rows, sum, store in turn); one token of 64 sequences x 8 heads 4.9 us, 512 tokens x 32 heads 8.0 us = 1.6 TB/s.
template <int DT>
__global__ __launch_bounds__(128) void kv_append_kernel(const KvItem *__restrict__ items, const KvSeq *__restrict__ seqs, KvShape s, KvAppend a)
{
    const KvItem it = items[blockIdx.x / s.n_kv];
    const int head = blockIdx.x % s.n_kv, which = wave_number(), lane = threadIdx.x % kWave;
    const int64_t entry = table_entry(s, seqs[it.s].seq, it.a, head);
    uint8_t *page = s.pool + (int64_t)s.table[entry] * s.page_bytes;
    const int D = s.D, t0 = it.b, n = it.c;
    const uint16_t *x = a.x[which] + (int64_t)it.d * a.stride[which] + (int64_t)head * D;
    const int64_t stride = a.stride[which];
    const int before = t0 > 0 ? s.exps[2 * entry + which] : kKvLowest;

    // 16 bytes a lane: D / 8 lanes to a row
    const int per_row = D / 8, rows_at_once = kWave / per_row, r0 = lane / per_row, c0 = lane % per_row * 8;
    const bool on = r0 < rows_at_once;
    uint32_t top = 0; // largest magnitude, as the bits of its 16-bit form (which order as the values do)
    constexpr int kAhead = 4; // rows of a lane that are loaded together (those behind the last: the last once more)
    u32x4 kept[kAhead] = {}; // ... of which a single round's stay for K's second pass
    for (int r = r0; on && r < n; r += kAhead * rows_at_once) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) kept[j] = *reinterpret_cast<const u32x4 *>(x + min(r + j * rows_at_once, n - 1) * stride + c0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, max(kept[j][k] & 0x7fffu, (kept[j][k] >> 16) & 0x7fffu));
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, kWave));
    const int e = max(before, exponent_of(widen<DT>((uint16_t)top)));
    const bool poison = e == kKvPoison;
    const float inverse = poison ? 0.0f : inverse_of(e);
    const bool grown = e != before;
    const float factor = shift_factor(before, e);

    if (which == 0) {
        // slot t of the block: granule t / 8, row t % 8
        auto row_at = [&](int t) { return page + (int64_t)(t / kKvGranule) * (2 * kKvGranule * D) + (t % kKvGranule) * D; };
        if (grown)
            for (int t = r0; on && t < t0; t += rows_at_once) {
                u32x2 *p = reinterpret_cast<u32x2 *>(row_at(t) + c0);
                u32x2 u = *p;
                u.x = shift_codes(u.x, factor);
                u.y = shift_codes(u.y, factor);
                *p = u;
            }
        for (int r = r0; on && r < n; r += kAhead * rows_at_once) {
            if (n > kAhead * rows_at_once)
#pragma unroll
                for (int j = 0; j < kAhead; ++j) kept[j] = *reinterpret_cast<const u32x4 *>(x + min(r + j * rows_at_once, n - 1) * stride + c0);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                uint32_t o[2] = {0, 0};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float v = widen<DT>((uint16_t)(kept[j][k / 2] >> (16 * (k % 2))));
                    if (!poison) o[k / 4] |= ((uint32_t)code_of(v, inverse) & 0xffu) << (8 * (k % 4));
                }
                if (r + j * rows_at_once < n) *reinterpret_cast<u32x2 *>(row_at(t0 + r + j * rows_at_once) + c0) = u32x2{o[0], o[1]};
            }
        }
    } else {
        const int first = grown ? 0 : t0 / kKvGranule, last = (t0 + n - 1) / kKvGranule;
        const int pairs = D / 2;
        for (int w = lane; w < pairs * (last - first + 1); w += kWave) {
            const int g = first + w / pairs, d = w % pairs * 2;
            u32x4 *p = reinterpret_cast<u32x4 *>(page + (int64_t)g * (2 * kKvGranule * D) + kKvGranule * D + d * kKvGranule);
            const int lo = g * kKvGranule, from = max(t0 - lo, 0), to = min(t0 + n - lo, kKvGranule); // its new tokens: [from, to)
            uint32_t u[4] = {0, 0, 0, 0}; // element d: slots 0 .. 3, 4 .. 7; element d + 1
            if (from > 0 || to < kKvGranule) {
                const u32x4 all = *p;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    u[k] = all[k];
                    const int mine = min(max(from - 4 * (k % 2), 0), 4); // slots before t0; those behind the new ones are nobody's
                    const uint32_t mask = mine == 4 ? 0xffffffffu : (1u << (8 * mine)) - 1;
                    if (grown) u[k] = (shift_codes(u[k], factor) & mask) | (u[k] & ~mask);
                }
            }
            uint32_t raw[kKvGranule];
#pragma unroll
            for (int t = 0; t < kKvGranule; ++t) raw[t] = *reinterpret_cast<const uint32_t *>(x + min(max(lo + t - t0, 0), n - 1) * stride + d);
#pragma unroll
            for (int t = 0; t < kKvGranule; ++t) {
                if (t < from || t >= to) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float v = widen<DT>((uint16_t)(raw[t] >> (16 * h)));
                    const uint32_t c = poison ? 0u : (uint32_t)code_of(v, inverse) & 0xffu;
                    uint32_t &word = u[2 * h + t / 4];
                    word = (word & ~(0xffu << (8 * (t % 4)))) | (c << (8 * (t % 4)));
                }
            }
            *p = u32x4{u[0], u[1], u[2], u[3]};
        }
    }
    if (lane == 0) s.exps[2 * entry + which] = (int8_t)e;
}

// ---------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------
// Matrix instruction 16 x 16 x 32 (f16): lane l = 16 g + n supplies k-values 8 g .. 8 g + 7 of row (first operand) or column
// (second) n, and receives rows 4 g .. 4 g + 3 of column n.
//
// A wavefront takes 32 tokens (four granules) and 16 columns (a column = a query row and one of the heads that share the
// cache's head) at a time, with the scores transposed: S' = K Q', so that a lane's scores are of ONE column.  Rows of S' may
// be any tokens: row 4 g + i of its half t is token 4 t + i of granule g, so that lane (g, n) ends with the scores of all eight tokens of
// granule g - the k-values it has to supply for O' = V' P', whose first operand is eight bytes of V: probabilities go
// from one product to the next in the registers where they are, and K and V come from memory straight
// into operands.  Codes become binary16 exactly (|c| <= 127); q in bfloat16 is scaled by a power of two of its own into the range of
// binary16, which keeps its eight bits down to 2^-28 of the row's largest.
//
// Softmax: with scores s (times log2 e) and V's exponents ev, u = max(ev - top, -100) for the largest exponent `top` of the part, the
// running maximum is of s + u, so that p = 2^(s + u - m) <= 1 is what the second product needs of V's units; the sum that
// divides takes p * 2^-u.  p is the one number that is rounded, since that product takes 16-bit operands: for few columns to 22 bits, as two of binary16, which costs
// half a percent where the cache's bytes are the bound (64 of 500 - 8000 tokens 123.9 us with one, 124.4 with two; 24 of 200 - 1500 60.0 / 60.4); for prompts to
// the 11 bits of one, since two take a quarter longer (chunks of 128 - 1024 behind up to 4096 tokens 438 us / 539, a prompt of 512 29.5 / 31.6) and the output's own
// rounding, to 11 or 8 bits, is as large.  p is taken 2^15 times as large (2^7 times for prompts, whose maximum may be 2^8 behind), the
// largest power that stays in range, so that binary16 has its 11 bits down to 2^-29 (2^-21) of the largest.
// The token whose s + u is m adds 2^-u >= 1 to the scores' sum, and one of equal score has p >= 2^-100, whatever exponents there are.  V of a block further below `top` is read in units of 2^(top - 100) instead of its own, which puts its elements off by less than 2^(top - 93).
// A block with an infinity or NaN in V has u = 0, and the columns that see any of its tokens - their limits are behind its first one - get NaN at the end: the
// scores' sum, which the weights are taken from, knows nothing of V.
__device__ __forceinline__ f32x4 mfma16(const f16x8 &a, const f16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// four codes -> binary16: 0x6400 | u is 1024 + u for a byte u; c + 128 = u
__device__ __forceinline__ void codes_to_f16(uint32_t u, half2_t &a, half2_t &b)
{
    u ^= 0x80808080u;
    const half2_t bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
    b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
}
__device__ __forceinline__ f16x8 codes_to_f16x8(uint32_t lo, uint32_t hi)
{
    half2_t r[4];
    codes_to_f16(lo, r[0], r[1]);
    codes_to_f16(hi, r[2], r[3]);
    return __builtin_shufflevector(__builtin_shufflevector(r[0], r[1], 0, 1, 2, 3), __builtin_shufflevector(r[2], r[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}

// Which element of a head the operands of step j hold in k-value i of lane group g: K's rows are read 16 bytes a lane, two
// steps at a time; the last step of an odd number reads 8.
template <int DB>
__device__ __forceinline__ int element_of(int j, int g)
{
    return j / 2 * 2 + 1 < DB ? j / 2 * 64 + 16 * g + 8 * (j % 2) : j * 32 + 8 * g;
}

// q of bfloat16 in the range of binary16: its largest magnitude has exponent bits x, and times 2^(141 - x) lies in [2^14, 2^15).  The power is kept
// where its inverse is a normal number too; an infinity or NaN stays what it is.
__device__ __forceinline__ int power_for_f16(uint32_t top)
{
    const int x = (int)(top >> 7);
    return x == 255 ? 0 : min(141 - x, 126);
}

// q of one column as second operands, element(j) on for step j, and the power of two to multiply its scores by.  Lanes that differ in the bits
// of LANES hold other elements of the same column.
template <int DT, int STEPS, int LANES, typename F>
__device__ __forceinline__ void load_column(const uint16_t *q, F element, f16x8 (&f)[STEPS], float &unit)
{
    unit = 1.0f;
    if constexpr (DT == SLORA_F16) {
#pragma unroll
        for (int j = 0; j < STEPS; ++j) f[j] = q ? __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4 *>(q + element(j))) : f16x8{};
    } else {
        u32x4 raw[STEPS];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            raw[j] = q ? *reinterpret_cast<const u32x4 *>(q + element(j)) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, max(raw[j][k] & 0x7fffu, (raw[j][k] >> 16) & 0x7fffu));
        }
#pragma unroll
        for (int x = 16; x < kWave; x *= 2)
            if (LANES & x) top = max(top, (uint32_t)__shfl_xor((int)top, x, kWave));
        const int up = power_for_f16(top);
        const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
        unit = __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int j = 0; j < STEPS; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) f[j][k] = (_Float16)(__uint_as_float((raw[j][k / 2] >> (16 * (k % 2))) << 16) * scale);
    }
}
template <int DT, int DB>
__device__ __forceinline__ void load_q(const uint16_t *q, int g, f16x8 (&f)[DB], float &unit)
{
    load_column<DT, DB, 48>(q, [=](int j) { return element_of<DB>(j, g); }, f, unit);
}
template <int DT, int DB>
__device__ __forceinline__ void load_q32(const uint16_t *q, int h, f16x8 (&f)[2 * DB], float &unit)
{
    load_column<DT, 2 * DB, 32>(q, [=](int j) { return 16 * j + 8 * h; }, f, unit);
}

// (the cache is read once)
__device__ __forceinline__ u32x4 load_once(const uint8_t *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}
// K of one token as first operands, from its row
template <int DB>
__device__ __forceinline__ void load_k(const uint8_t *row, int g, u32x4 (&raw)[(DB + 1) / 2])
{
#pragma unroll
    for (int p = 0; p < (DB + 1) / 2; ++p) {
        if (2 * p + 1 < DB) {
            raw[p] = load_once(row + 64 * p + 16 * g);
        } else {
            const u32x2 u = *reinterpret_cast<const u32x2 *>(row + 64 * p + 8 * g);
            raw[p] = u32x4{u.x, u.y, 0u, 0u};
        }
    }
}
template <int DB>
__device__ __forceinline__ f16x8 k_operand(const u32x4 (&raw)[(DB + 1) / 2], int j)
{
    return j % 2 ? codes_to_f16x8(raw[j / 2].z, raw[j / 2].w) : codes_to_f16x8(raw[j / 2].x, raw[j / 2].y);
}

constexpr int kKvFar = 100; // see above
constexpr int kFewUp = 15, kManyUp = 7; // powers of two of p in the second product

// the largest of the lanes' numbers, without LDS: rows of 16, then what the rows before have found
__device__ __forceinline__ int wave_max(int v)
{
#define SLORA_STEP(control) v = max(v, __builtin_amdgcn_update_dpp(v, v, control, 0xf, 0xf, false))
    SLORA_STEP(0x111); // row_shr 1, 2, 4, 8
    SLORA_STEP(0x112);
    SLORA_STEP(0x114);
    SLORA_STEP(0x118);
    SLORA_STEP(0x142); // row_bcast 15, 31
    SLORA_STEP(0x143);
#undef SLORA_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

// what a part's exponents of V are taken against
struct Units {
    int top;     // the largest of them
    int spoiled; // the first block of the part that holds an infinity or NaN, if any
    __device__ __forceinline__ int of(int ev) const { return ev == kKvPoison ? 0 : max(ev - top, -kKvFar); }
    // what a column's sums of 2^up p V are multiplied by (limit: tokens that it sees; a block's first token: N of them before each)
    __device__ __forceinline__ float scale(float by, int up, int limit, int N, int block0) const
    {
        return spoiled < INT32_MAX && limit > (block0 + spoiled) * N ? __uint_as_float(0x7fc00000u) : by * unit_of(top - up);
    }
};

// Pages and exponents of the blocks of a part, in LDS
struct PartPages {
    int32_t page[kKvPartBlocks];
    int16_t e[kKvPartBlocks]; // K in the low byte, V above
};
__device__ __forceinline__ void load_pages(PartPages &pp, const KvShape &s, int seq, int head, int block0, int blocks)
{
    for (int i = threadIdx.x; i < blocks; i += blockDim.x) {
        const int64_t entry = table_entry(s, seq, block0 + i, head);
        pp.page[i] = s.table[entry];
        pp.e[i] = reinterpret_cast<const int16_t *>(s.exps)[entry];
    }
}
// (every wavefront for itself, behind the barrier that ends load_pages)
__device__ __forceinline__ Units units_of(const PartPages &pp, int blocks)
{
    const int lane = threadIdx.x % kWave;
    int top = kKvLowest, spoiled = INT32_MAX;
    for (int i0 = 0; i0 < blocks; i0 += kWave) {
        const int ev = i0 + lane < blocks ? pp.e[i0 + lane] >> 8 : kKvLowest;
        const uint64_t bad = __ballot(ev == kKvPoison);
        if (bad) spoiled = min(spoiled, i0 + (int)__ffsll((unsigned long long)bad) - 1);
        top = max(top, ev == kKvPoison ? kKvLowest : ev);
    }
    return {wave_max(top), spoiled};
}

// 1 / the scores' sum of a row.  One that sees no token is 0; one that does and has none in its sum has scores of -infinity alone, and no softmax.
__device__ __forceinline__ float inverse_sum(float l, bool sees) { return l != 0.0f ? 1.0f / l : sees ? __uint_as_float(0x7fc00000u) : 0.0f; }

// A part leaves its own average of V, whose units are its own, and {m, l}, its scores' sum as l * 2^m: l below 2^65 keeps l * 2^(m - the largest m) a
// normal number wherever it matters (its u may have made it 2^100 times its share).
__device__ __forceinline__ void put_sum(float *to, float m, float l)
{
    const bool large = l >= 0x1p64f;
    to[0] = large ? m + 64.0f : m;
    to[1] = large ? l * 0x1p-64f : l;
}

// A workgroup = one item: up to 16 columns x a part of the sequence; the wavefronts take chunks of 32 tokens in turn, keep their own
// maxima, sums and O', and are put together in LDS at the end.
// Bound: HBM, from which the cache comes once, with non-temporal loads (645 MB of 64 sequences, 8 heads: 115 us = 5.6 TB/s, with plain loads 125; 227 MB of
// 24 sequences, 40 heads: 46 us = 4.9 TB/s); a single sequence of 701 tokens takes 5.6 us, the chain of page, K, score, sum.  Vector units 43 - 45 %, matrix
// units 9 - 10 % busy even where one column of sixteen is in use, so there is no kernel of its own for one.
template <int DT, int DB>
__global__ __launch_bounds__(kKvFewThreads, DB <= 4 ? 3 : DB == 6 ? 2 : 1) void kv_attend_few_kernel(const KvItem *__restrict__ items, const KvSeq *__restrict__ seqs, KvShape s, KvAttend a)
{
    constexpr int D = DB * 32, kWaves = kKvFewThreads / kWave;
    __shared__ PartPages pp;
    __shared__ float merge_ml[kWaves][kKvFewCols][2];
    __shared__ float merge_o[kWaves][kKvFewCols][D];
    const KvItem it = items[blockIdx.x / s.n_kv];
    const int head = blockIdx.x % s.n_kv;
    const KvSeq q = seqs[it.s];
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    const int gpb = s.N / kKvGranule;

    // this lane's column, and how many tokens it sees
    const int col = it.a + n, row = col / s.G;
    const bool real = n < it.b;
    const int old = q.len - q.rows;
    const int limit = !real ? 0 : a.causal ? min(old + row + 1, q.len) : q.len;
    const int last_row = (it.a + it.b - 1) / s.G;
    const int tokens = a.causal ? min(old + last_row + 1, q.len) : q.len;
    const int g1 = min(it.d, (max(tokens, 0) + kKvGranule - 1) / kKvGranule), g0 = it.c;
    const int block0 = g0 / gpb, base = block0 * gpb;
    const int blocks = g1 > g0 ? (g1 - 1) / gpb + 1 - block0 : 0;
    load_pages(pp, s, q.seq, head, block0, blocks);

    f16x8 qf[DB];
    float unit;
    const int qhead = head * s.G + col % s.G;
    load_q<DT, DB>(real ? a.q + (int64_t)(q.row0 + row) * a.q_stride + (int64_t)qhead * D : nullptr, g, qf, unit);
    unit *= a.scale;
    __syncthreads();

    Units units;
    f32x4 o[2 * DB];
#pragma unroll
    for (int k = 0; k < 2 * DB; ++k) o[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;

    // of the granules of a chunk, a lane reads K rows of number n / 4 (4 t + n % 4 of it) and V of number g, whose scores it gets
    u32x4 kr[2][(DB + 1) / 2], vr[DB];
    int e_next = 0;
    auto fetch = [&](int gr) {
        const int gk = min(gr + n / 4, g1 - 1) - base, gv = min(gr + g, g1 - 1) - base;
        const int bk = (int)kv_div((uint32_t)gk, s.div_b), bv = (int)kv_div((uint32_t)gv, s.div_b);
        const uint8_t *pk = s.pool + (int64_t)pp.page[bk] * s.page_bytes + (int64_t)(gk - bk * gpb) * (2 * kKvGranule * D) + (n % 4) * D;
        const uint8_t *pv = s.pool + (int64_t)pp.page[bv] * s.page_bytes + (int64_t)(gv - bv * gpb) * (2 * kKvGranule * D) + kKvGranule * D + n * 16;
        load_k<DB>(pk, g, kr[0]);
        load_k<DB>(pk + 4 * D, g, kr[1]);
#pragma unroll
        for (int k = 0; k < DB; ++k) vr[k] = load_once(pv + k * 256);
        e_next = pp.e[bv];
    };
    constexpr int kStep = kWaves * (kKvChunk / kKvGranule);
    auto work = [&](int gr, auto more) {
        // operands of this chunk, then the next chunk's loads (not behind a branch: the compiler would wait for all loads where it joins)
        f32x4 sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < DB; ++j) sc[t] = mfma16(k_operand<DB>(kr[t], j), qf[j], sc[t]);
        }
        u32x4 v[DB];
#pragma unroll
        for (int k = 0; k < DB; ++k) v[k] = vr[k];
        const int ek = (int8_t)(e_next & 0xff), ev = e_next >> 8;
        const int token = (gr + g) * kKvGranule;
        const int bound = min(limit, g1 * kKvGranule) - token; // tokens of this lane's granule that its column sees
        if constexpr (more.value) fetch(gr + kStep);

        const int u = units.of(ev);
        const float f = unit * unit_of(ek), add = (float)u;
        float t[8], top = -INFINITY;
        if (a.scores && q.score0 >= 0) {
            float *at = a.scores + (q.score0 + ((int64_t)head * (q.rows * s.G) + col) * (int64_t)((q.len + 7) / 8 * 8)) + token;
            f32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = i < bound ? sc[0][i] * f : -INFINITY;
                hi[i] = i + 4 < bound ? sc[1][i] * f : -INFINITY;
            }
            if (real && token < q.len) {
                *reinterpret_cast<f32x4 *>(at) = lo;
                *reinterpret_cast<f32x4 *>(at + 4) = hi;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t[i] = i < bound ? __builtin_fmaf(sc[i / 4][i % 4], f, add) : -INFINITY;
            top = fmaxf(top, t[i]);
        }
        top = fmaxf(top, across_16(top));
        top = fmaxf(top, across_32(top));
        const float m_new = fmaxf(m, top), m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float keep = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        float sum = 0.0f;
        f16x8 p, rest;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = __builtin_amdgcn_exp2f(t[i] - (m_use - kFewUp));
            sum += x;
            p[i] = (_Float16)x;
            rest[i] = (_Float16)(x - (float)p[i]);
        }
        l = __builtin_fmaf(l, keep, sum * unit_of(-u - kFewUp));
        if (__any(keep != 1.0f)) {
#pragma unroll
            for (int k = 0; k < 2 * DB; ++k) o[k] *= keep;
        }
        // element 32 k + 2 m + h of row m of o[2 k + h]
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            const f16x8 v0 = codes_to_f16x8(v[k].x, v[k].y), v1 = codes_to_f16x8(v[k].z, v[k].w);
            o[2 * k] = mfma16(v0, p, o[2 * k]);
            o[2 * k + 1] = mfma16(v1, p, o[2 * k + 1]);
            o[2 * k] = mfma16(v0, rest, o[2 * k]);
            o[2 * k + 1] = mfma16(v1, rest, o[2 * k + 1]);
        }
    };
    int gr = g0 + wave * (kKvChunk / kKvGranule);
    if (gr < g1) fetch(gr);
    units = units_of(pp, blocks); // (while the first chunk is on its way)
    if (gr < g1) {
        for (; gr + kStep < g1; gr += kStep) work(gr, std::true_type{});
        work(gr, std::false_type{});
    }
    l += across_16(l);
    l += across_32(l);

    if (real) {
        if (g == 0) {
            merge_ml[wave][n][0] = m;
            merge_ml[wave][n][1] = l;
        }
#pragma unroll
        for (int k = 0; k < DB; ++k) // elements 32 k + 8 g .. + 7
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                merge_o[wave][n][32 * k + 8 * g + 2 * i] = o[2 * k][i];
                merge_o[wave][n][32 * k + 8 * g + 2 * i + 1] = o[2 * k + 1][i];
            }
    }
    __syncthreads();
    for (int w = (int)threadIdx.x; w < it.b * (D / 8); w += kKvFewThreads) {
        const int c = w / (D / 8), d = w % (D / 8) * 8;
        float top = -INFINITY, total = 0.0f, sum[8] = {};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) top = fmaxf(top, merge_ml[k][c][0]);
        const float use = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float x = __builtin_amdgcn_exp2f(merge_ml[k][c][0] - use);
            total = __builtin_fmaf(merge_ml[k][c][1], x, total);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(merge_o[k][c][d + i], x, sum[i]);
        }
        const int r = (it.a + c) / s.G;
        const int sees = a.causal ? min(old + r + 1, q.len) : q.len;
        const float by = inverse_sum(total, it.poff < 0 && sees > 0), scale = units.scale(by, kFewUp, sees, s.N, block0);
        if (it.poff >= 0) {
            const int64_t at = (int64_t)(it.poff + c) * s.n_kv + head;
#pragma unroll
            for (int i = 0; i < 8; ++i) a.part_o[at * D + d + i] = sum[i] * scale;
            if (d == 0) put_sum(a.part_ml + 2 * at, top, total);
        } else {
            const int h = head * s.G + (it.a + c) % s.G;
            u32x4 u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = (uint32_t)narrow<DT>(sum[2 * i] * scale) | ((uint32_t)narrow<DT>(sum[2 * i + 1] * scale) << 16);
            *reinterpret_cast<u32x4 *>(a.out + (int64_t)(q.row0 + r) * a.out_stride + (int64_t)h * D + d) = u;
            if (d == 0) {
                float *st = a.stat + 2 * ((int64_t)(q.row0 + r) * s.n_kv * s.G + h);
                st[0] = use;
                st[1] = by;
            }
        }
    }
}

// Many columns (prompts).  Matrix instruction 32 x 32 x 16: lane l = 32 h + n supplies k-values 8 h .. 8 h + 7 of row or column n and receives
// rows 8 b + 4 h + i of column n (register 4 b + i).
//
// A workgroup = an item of up to 128 columns, 32 to a wavefront, that walk the tokens in tiles of 64 together.  A tile's codes are turned into
// binary16 once, on the way into LDS: K in units of 8 elements of a token, [unit][token] (tokens of a granule change
// places from one pair of units to the next, so that the eight lanes that write a token are in different banks), V in units of 8 tokens of an element as its granules hold them - so that every
// operand is one read of 16 bytes, lane by lane in order.  While one tile is worked on, the next one's loads are under way; it
// goes into the other buffer afterwards, and one barrier ends the round.
//
// As above the scores are transposed, and which token is which row is chosen so that a lane's scores are the k-values that it
// has to supply next: row 16 s + 8 b + 4 h + i of a half of the tile is its token 16 s + 8 h + 4 b + i, of granule 2 s + h.
// The maximum is only raised when a score exceeds it by kSlack: until then probabilities stay below 2^kSlack, 2^15 with the power that they are taken at.
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma32(const f16x8 &a, const f16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kManyTile = kKvManyTile, kManyGranules = kManyTile / kKvGranule;
constexpr float kSlack = 8.0f;

// Bound: the vector units, 12 of whose instructions go beside each matrix instruction (over half of all cycles, at four an instruction; matrix units 35 %): a chunk of 512 behind 30000 tokens, 64 heads 680 us = 750 TFLOP/s, chunks of 128 - 1024 behind up to 4096 426 - 440 us.
// Two workgroups share a compute unit up to 128 elements a head, so that one's products run beside the other's softmax.
template <int DB>
struct ManyLds {
    static constexpr int kUnits = kManyTile * DB * 4; // of 16 bytes, K's or V's of a tile
    u32x4 k[2][kUnits], v[2][kUnits];
    float unit[2][kManyGranules], add[2][kManyGranules], less[2][kManyGranules]; // 2^ek, u + kManyUp, 2^-(u + kManyUp) of each granule
    PartPages pages;
};

template <int DT, int DB>
__global__ __launch_bounds__(kKvManyThreads, DB <= 4 ? 2 : 1) void kv_attend_many_kernel(const KvItem *__restrict__ items, const KvSeq *__restrict__ seqs, KvShape s, KvAttend a)
{
    constexpr int D = DB * 32, kSteps = 2 * DB;
    extern __shared__ u32x4 lds_bytes[];
    ManyLds<DB> &lds = *reinterpret_cast<ManyLds<DB> *>(lds_bytes);
    const KvItem it = items[blockIdx.x / s.n_kv];
    const int head = blockIdx.x % s.n_kv;
    const KvSeq q = seqs[it.s];
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 32, h = lane / 32;
    const int gpb = s.N / kKvGranule, old = q.len - q.rows;

    const int col = it.a + wave * 32 + n, row = col / s.G;
    const bool real = wave * 32 + n < it.b;
    const int last_row = (it.a + it.b - 1) / s.G;
    const int limit = !real ? q.len : a.causal ? min(old + row + 1, q.len) : q.len; // tokens that this lane's column sees
    const int tokens = a.causal ? min(old + last_row + 1, q.len) : q.len;
    const int g0 = it.c, g1 = min(it.d, (max(tokens, 0) + kKvGranule - 1) / kKvGranule);
    // of this wavefront's columns: what all of them see, what any sees
    const int all_see = a.causal ? min(old + (it.a + min(wave * 32, it.b - 1)) / s.G + 1, q.len) : q.len;
    const int any_sees = wave * 32 >= it.b ? 0 : a.causal ? min(old + (it.a + min(wave * 32 + 31, it.b - 1)) / s.G + 1, q.len) : q.len;
    const int block0 = g0 / gpb, base = block0 * gpb;
    const int blocks = g1 > g0 ? (g1 - 1) / gpb + 1 - block0 : 0;
    load_pages(lds.pages, s, q.seq, head, block0, blocks);

    f16x8 qf[kSteps];
    float unit;
    const int qhead = head * s.G + col % s.G;
    load_q32<DT, DB>(real ? a.q + (int64_t)(q.row0 + row) * a.q_stride + (int64_t)qhead * D : nullptr, h, qf, unit);
    unit *= a.scale;
    __syncthreads();

    const Units units = units_of(lds.pages, blocks);

    f32x16 o[DB];
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[k][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    // eight lanes that write every other unit are in different banks
    auto v_place = [](int unit) { return unit ^ (unit >> 3 & 1); };
    // a tile's pieces of 16 bytes, D to a granule (K's first), 256 at a time
    u32x4 raw[DB];
    auto fetch = [&](int g) {
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            const int u = threadIdx.x + i * kKvManyThreads, gk = min(g + u / D, g1 - 1) - base;
            const int b = (int)kv_div((uint32_t)gk, s.div_b);
            raw[i] = *reinterpret_cast<const u32x4 *>(s.pool + (int64_t)lds.pages.page[b] * s.page_bytes + (int64_t)(gk - b * gpb) * (2 * kKvGranule * D) + u % D * 16);
        }
    };
    auto put = [&](int buffer, int g) {
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            const int u = threadIdx.x + i * kKvManyThreads, w = u % D;
            const u32x4 lo = __builtin_bit_cast(u32x4, codes_to_f16x8(raw[i].x, raw[i].y)), hi = __builtin_bit_cast(u32x4, codes_to_f16x8(raw[i].z, raw[i].w));
            if (w < D / 2) { // 16 elements of a token: units 2 c, 2 c + 1
                const int token = u / D * kKvGranule + w / (D / 16), c = w % (D / 16), at = token ^ (c % 8);
                lds.k[buffer][2 * c * kManyTile + at] = lo;
                lds.k[buffer][(2 * c + 1) * kManyTile + at] = hi;
            } else { // two elements' eight tokens
                const int at = u / D * D + 2 * (w - D / 2);
                lds.v[buffer][v_place(at)] = lo;
                lds.v[buffer][v_place(at + 1)] = hi;
            }
        }
        if (threadIdx.x < kManyGranules) {
            const int gk = min(g + (int)threadIdx.x, g1 - 1) - base, e = lds.pages.e[kv_div((uint32_t)gk, s.div_b)];
            const int ek = (int8_t)(e & 0xff), ev = e >> 8;
            lds.unit[buffer][threadIdx.x] = unit_of(ek);
            const int u = units.of(ev) + kManyUp;
            lds.add[buffer][threadIdx.x] = (float)u;
            lds.less[buffer][threadIdx.x] = unit_of(-u);
        }
    };
    // this lane's token in row n of a half of the tile, and its place in LDS for units 2 s + h, s even and odd
    const int token_n = n / 16 * 16 + n / 4 % 2 * 8 + n / 8 % 2 * 4 + n % 4;
    if (g1 > g0) {
        fetch(g0);
        put(0, g0);
    }
    __syncthreads();
    int buffer = 0;
    for (int g = g0; g < g1; g += kManyGranules, buffer ^= 1) {
        const bool more = g + kManyGranules < g1;
        if (more) fetch(g + kManyGranules);
        const int first = g * kKvGranule;
        if (first < any_sees) {
            // Operands are read a group of steps ahead of the products that take them (left to itself the compiler reads each one right before,
            // and waits), and the halves take turns, so that a product does not wait for the one before.
            f32x16 sc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = 0.0f;
            constexpr int kGroup = 2, kGroups = kSteps / kGroup;
            f16x8 kf[2][kGroup][2];
            auto read_k = [&](int j0, f16x8 (&to)[kGroup][2]) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
#pragma unroll
                    for (int t = 0; t < 2; ++t) // unit 2 j + h: c = j
                        to[j][t] = __builtin_bit_cast(f16x8, lds.k[buffer][(2 * (j0 + j) + h) * kManyTile + t * 32 + (token_n ^ ((j0 + j) % 8))]);
            };
            read_k(0, kf[0]);
#pragma unroll
            for (int b = 0; b < kGroups; ++b) {
                if (b + 1 < kGroups) read_k((b + 1) * kGroup, kf[(b + 1) % 2]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
#pragma unroll
                    for (int t = 0; t < 2; ++t) sc[t] = mfma32(kf[b % 2][j][t], qf[b * kGroup + j], sc[t]);
                __builtin_amdgcn_sched_barrier(0);
            }
            // registers 8 s .. 8 s + 7 of half t: granule 4 t + 2 s + h.  Scores from here on are less the maximum so far.
            const float so_far = m == -INFINITY ? 0.0f : m;
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float f = unit * lds.unit[buffer][4 * t + 2 * r + h], add = lds.add[buffer][4 * t + 2 * r + h] - so_far;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sc[t][8 * r + i] = __builtin_fmaf(sc[t][8 * r + i], f, add);
                }
            if (first + kManyTile > min(all_see, g1 * kKvGranule)) {
                const int bound = min(limit, g1 * kKvGranule) - first - 8 * h;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t * 32 + i / 8 * 16 + i % 8 >= bound) sc[t][i] = -INFINITY;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[t][i]);
            top = fmaxf(top, across_32(top));
            const bool raise = top > kSlack + kManyUp || (m == -INFINITY && top > -INFINITY);
            if (__any(raise)) {
                const float by = raise ? top - kManyUp : 0.0f, m_new = raise ? so_far + by : m;
                const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(-by); // (nothing has been added up before the first maximum)
                m = m_new;
                l *= keep;
#pragma unroll
                for (int k = 0; k < DB; ++k)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[k][i] *= keep;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[t][i] -= by;
            }
            f16x8 p[2][2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = __builtin_amdgcn_exp2f(sc[t][8 * r + i]);
                        sum += x;
                        p[t][r][i] = (_Float16)x;
                    }
                    l = __builtin_fmaf(sum, lds.less[buffer][4 * t + 2 * r + h], l);
                }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int k = 0; k < DB; ++k)
                        o[k] = mfma32(__builtin_bit_cast(f16x8, lds.v[buffer][(4 * t + 2 * r + h) * D + 32 * k + v_place(n)]), p[t][r], o[k]);
        }
        if (more) put(buffer ^ 1, g + kManyGranules);
        __syncthreads();
    }
    l += across_32(l);
    if (!real) return;
    // elements 32 k + 8 b + 4 h + i of column n are register 4 b + i of o[k]
    const float by = inverse_sum(l, it.poff < 0 && limit > 0), scale = units.scale(by, kManyUp, limit, s.N, block0);
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[k][i] *= scale;
    if (it.poff >= 0) {
        const int64_t at = (int64_t)(it.poff + wave * 32 + n) * s.n_kv + head;
#pragma unroll
        for (int k = 0; k < DB; ++k)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<f32x4 *>(a.part_o + at * D + 32 * k + 8 * b + 4 * h) = f32x4{o[k][4 * b], o[k][4 * b + 1], o[k][4 * b + 2], o[k][4 * b + 3]};
        if (h == 0) put_sum(a.part_ml + 2 * at, m, l);
        return;
    }
    uint16_t *out = a.out + (int64_t)(q.row0 + row) * a.out_stride + (int64_t)qhead * D;
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *reinterpret_cast<u32x2 *>(out + 32 * k + 8 * b + 4 * h) =
                u32x2{(uint32_t)narrow<DT>(o[k][4 * b]) | (uint32_t)narrow<DT>(o[k][4 * b + 1]) << 16,
                      (uint32_t)narrow<DT>(o[k][4 * b + 2]) | (uint32_t)narrow<DT>(o[k][4 * b + 3]) << 16};
    if (h == 0) {
        float *st = a.stat + 2 * ((int64_t)(q.row0 + row) * s.n_kv * s.G + qhead);
        st[0] = m == -INFINITY ? 0.0f : m;
        st[1] = by;
    }
}

// Parts of a column put together, in the order of the sequence.  W = 4: a workgroup per column, whose wavefronts take parts in turn and are
// added in LDS; W = 1, where there are few parts: a wavefront per column.
// Bound: latency; 24 x 40 columns of up to 4 parts 4.7 us, 16 x 8 of up to 64 parts 8.4 us.
template <int DT, int DB, int W>
__global__ __launch_bounds__(256) void kv_join_kernel(const KvItem *__restrict__ items, const KvSeq *__restrict__ seqs, KvShape s, KvAttend a)
{
    constexpr int D = DB * 32, kPer = (D + kWave - 1) / kWave; // elements of a lane
    __shared__ float merge[W][kPer * kWave + 1];
    const KvItem it = items[blockIdx.x / s.n_kv];
    const int head = blockIdx.x % s.n_kv, wave = wave_number() % W, lane = threadIdx.x % kWave;
    const int c = (int)blockIdx.y * (4 / W) + wave_number() / W;
    if (c >= it.b) return;
    const KvSeq q = seqs[it.s];
    const int64_t first = (int64_t)(it.poff + c) * s.n_kv + head, step = (int64_t)it.b * s.n_kv;
    float top = -INFINITY;
    for (int k = lane; k < it.c; k += kWave) top = fmaxf(top, a.part_ml[2 * (first + k * step)]);
#pragma unroll
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, kWave));
    const float use = top == -INFINITY ? 0.0f : top;
    float total = 0.0f, sum[kPer] = {};
    constexpr int kAhead = 4;
    for (int k0 = wave; k0 < it.c; k0 += kAhead * W) {
        float x[kAhead], o[kAhead][kPer];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int k = k0 + j * W;
            const int64_t at = first + min(k, it.c - 1) * step;
            x[j] = k < it.c ? a.part_ml[2 * at + 1] * __builtin_amdgcn_exp2f(a.part_ml[2 * at] - use) : 0.0f; // its share of the scores' sum
#pragma unroll
            for (int i = 0; i < kPer; ++i) o[j][i] = a.part_o[at * D + min(lane + 64 * i, D - 1)];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (k0 + j * W >= it.c) break;
            total += x[j];
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum[i] = __builtin_fmaf(o[j][i], x[j], sum[i]);
        }
    }
    if constexpr (W > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) merge[wave][lane + 64 * i] = sum[i];
        if (lane == 0) merge[wave][kPer * kWave] = total;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            total += merge[w][kPer * kWave];
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum[i] += merge[w][lane + 64 * i];
        }
    }
    const int r = (it.a + c) / s.G;
    const float by = inverse_sum(total, (a.causal ? min(q.len - q.rows + r + 1, q.len) : q.len) > 0);
    const int h = head * s.G + (it.a + c) % s.G;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (lane + 64 * i < D) a.out[(int64_t)(q.row0 + r) * a.out_stride + (int64_t)h * D + lane + 64 * i] = narrow<DT>(sum[i] * by);
    if (lane == 0) {
        float *st = a.stat + 2 * ((int64_t)(q.row0 + r) * s.n_kv * s.G + h);
        st[0] = use;
        st[1] = by;
    }
}

// ---------------------------------------------------------------------------------------
// what cached tokens draw
// ---------------------------------------------------------------------------------------
// ... from scores that attention left, of sequences with few columns: a thread per token.  Scores of tokens that a column does not see, and of
// those behind the last that any sees, are not read.
// 24 sequences of 200 - 1500 tokens, 40 heads 6.0 us; computed again from K (as kv_weights_kernel does) it was 36.
__global__ __launch_bounds__(256) void kv_weights_few_kernel(const KvSeq *__restrict__ seqs, KvShape s, KvAttend a, KvWeights out)
{
    const KvSeq q = seqs[blockIdx.z];
    const int head = blockIdx.y, t = blockIdx.x * 256 + threadIdx.x, cols = q.rows * s.G;
    if (t >= q.len || q.score0 < 0) return;
    const int old = q.len - q.rows;
    const int64_t stride = (q.len + 7) / 8 * 8;
    const float *score = a.scores + q.score0 + (int64_t)head * cols * stride + t;
    float v = 0.0f;
    for (int c = 0; c < cols; ++c) {
        const int row = c / s.G, h = head * s.G + c % s.G;
        const float *st = a.stat + 2 * ((int64_t)(q.row0 + row) * s.n_kv * s.G + h);
        if (!a.causal || t <= old + row) v = __builtin_fmaf(__builtin_amdgcn_exp2f(score[c * stride] - st[0]), st[1], v);
    }
    const int64_t at = ((int64_t)q.seq * s.n_kv + head) * s.max_tokens + t;
    if (t < old)
        v += out.w_in[at];
    else
        out.pos[at] = q.seen - q.rows + t - old;
    out.w_out[at] = v;
}

// ... of many columns: the scores once more, from the maxima and sums that attention left.  A wavefront has the K of 32 tokens in registers (row
// 8 b + 4 h + i of the 32 x 32 instruction is its token of that number, of granule b); the workgroup's four go through the columns together,
// 32 at a time, which are put into LDS as binary16 while the ones before are worked on.  A lane adds up its tokens over its column of
// every tile; the 32 columns are added at the end.
// Bound: vector units (an exponential and two products for each score); a chunk of 512 behind 30000 tokens, 64 heads 605 us beside attention's 680.
template <int DB>
struct WeightsLds {
    u32x4 q[2][DB * 4 * 32]; // [8 elements][column]
    float unit[2][32], m[2][32], by[2][32]; // of each column: what its scores are multiplied by, maximum, 1 / sum
    int limit[2][32];                       // tokens it sees
};
template <int DT, int DB>
__global__ __launch_bounds__(256) void kv_weights_kernel(const KvSeq *__restrict__ seqs, KvShape s, KvAttend a, KvWeights out)
{
    constexpr int D = DB * 32, kSteps = 2 * DB;
    __shared__ WeightsLds<DB> lds;
    const KvSeq q = seqs[blockIdx.z];
    if (q.score0 >= 0) return; // (kv_weights_few_kernel's)
    const int head = blockIdx.y, wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 32, h = lane / 32;
    const int first = blockIdx.x * 128, token0 = first + wave * 32, granules = (q.len + kKvGranule - 1) / kKvGranule;
    if (first >= q.len) return;
    const int gpb = s.N / kKvGranule, old = q.len - q.rows, cols = q.rows * s.G;
    f16x8 kf[kSteps];
    float f[4];
    {
        auto block_of = [&](int g) { return (int)kv_div((uint32_t)g, s.div_b); };
        const int g = min(token0 / kKvGranule + n / kKvGranule, granules - 1), b = block_of(g);
        const uint8_t *row = s.pool + (int64_t)s.table[table_entry(s, q.seq, b, head)] * s.page_bytes + (int64_t)(g - b * gpb) * (2 * kKvGranule * D) + n % kKvGranule * D;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const u32x2 u = *reinterpret_cast<const u32x2 *>(row + 16 * j + 8 * h);
            kf[j] = codes_to_f16x8(u.x, u.y);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = unit_of(s.exps[2 * table_entry(s, q.seq, block_of(min(token0 / kKvGranule + k, granules - 1)), head)]);
    }
    // columns change places by the eighth of the elements that a unit is of: the eight threads that write a column are in different banks
    auto turn = [](int unit) { return unit * 64 / D % 8; };
    // a thread's share of a tile of columns: an eighth of one of them
    const int column = threadIdx.x / 8, part = threadIdx.x % 8;
    u32x2 raw[DB];
    float m_next = 0.0f, by_next = 0.0f;
    int limit_next = 0;
    auto fetch = [&](int c0) {
        const int col = c0 + column, row = col / s.G, qhead = head * s.G + col % s.G;
        const bool real = col < cols;
        const uint16_t *x = a.q + (int64_t)(q.row0 + (real ? row : 0)) * a.q_stride + (int64_t)(real ? qhead : head * s.G) * D + part * (D / 8);
#pragma unroll
        for (int k = 0; k < DB; ++k) raw[k] = real ? *reinterpret_cast<const u32x2 *>(x + 4 * k) : u32x2{0u, 0u};
        const float *st = a.stat + 2 * ((int64_t)(q.row0 + (real ? row : 0)) * s.n_kv * s.G + (real ? qhead : head * s.G));
        m_next = real ? st[0] : 0.0f;
        by_next = real ? st[1] : 0.0f;
        limit_next = !real ? 0 : a.causal ? min(old + row + 1, q.len) : q.len;
    };
    auto put = [&](int buffer) {
        float unit = 1.0f, scale = 1.0f;
        if constexpr (DT == SLORA_BF16) { // as load_column
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < DB; ++k) top = max(max(top, max(raw[k].x & 0x7fffu, (raw[k].x >> 16) & 0x7fffu)), max(raw[k].y & 0x7fffu, (raw[k].y >> 16) & 0x7fffu));
#pragma unroll
            for (int x = 1; x < 8; x *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, x, kWave));
            const int up = power_for_f16(top);
            scale = __uint_as_float((uint32_t)(127 + up) << 23);
            unit = __uint_as_float((uint32_t)(127 - up) << 23);
        }
#pragma unroll
        for (int k = 0; k < DB; ++k) { // elements e .. e + 3
            const int e = part * (D / 8) + 4 * k;
            u32x2 v = raw[k];
            if constexpr (DT == SLORA_BF16) {
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    v[w] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)(__uint_as_float(raw[k][w] << 16) * scale), (_Float16)(__uint_as_float(raw[k][w] & 0xffff0000u) * scale)});
            }
            reinterpret_cast<u32x2 *>(&lds.q[buffer][e / 8 * 32 + (column ^ turn(e / 8))])[e / 4 % 2] = v;
        }
        if (part == 0) {
            lds.unit[buffer][column] = unit * a.scale;
            lds.m[buffer][column] = m_next;
            lds.by[buffer][column] = by_next;
            lds.limit[buffer][column] = limit_next;
        }
    };
    float w[16] = {};
    // rows before the workgroup's first token see none of its tokens
    int c0 = a.causal ? max(first - old, 0) * s.G / 32 * 32 : 0, buffer = 0;
    if (c0 < cols) {
        fetch(c0);
        put(0);
    }
    __syncthreads();
    for (; c0 < cols; c0 += 32, buffer ^= 1) {
        if (c0 + 32 < cols) fetch(c0 + 32);
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) sc = mfma32(kf[j], __builtin_bit_cast(f16x8, lds.q[buffer][(2 * j + h) * 32 + (n ^ turn(2 * j + h))]), sc);
        const float unit = lds.unit[buffer][n], m = lds.m[buffer][n], by = lds.by[buffer][n];
        const int limit = lds.limit[buffer][n];
        // (what a column does not see is left out, not multiplied by 0: its score may be anything, and its sum may be NaN)
        auto add = [&](auto all) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * k + i], unit * f[k], -m)), sum = __builtin_fmaf(p, by, w[4 * k + i]);
                    w[4 * k + i] = all.value || token0 + 8 * k + 4 * h + i < limit ? sum : w[4 * k + i];
                }
        };
        if (__all(limit >= token0 + 32))
            add(std::true_type{});
        else
            add(std::false_type{});
        if (c0 + 32 < cols) put(buffer ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int x = 16; x; x >>= 1) w[i] += __shfl_xor(w[i], x, kWave);
    if (n >= 16) return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v = n == i ? w[i] : v;
    const int token = token0 + 8 * (n / 4) + 4 * h + n % 4;
    if (token >= q.len) return;
    const int64_t at = ((int64_t)q.seq * s.n_kv + head) * s.max_tokens + token;
    if (token < old)
        v += out.w_in[at];
    else
        out.pos[at] = q.seen - q.rows + token - old;
    out.w_out[at] = v;
}

// ---------------------------------------------------------------------------------------
// eviction
// ---------------------------------------------------------------------------------------
// numbers in the order of the weights: recent tokens above everything, then NaN, then values; -0 is 0
__device__ __forceinline__ uint32_t rank_of(float w, int32_t pos, int32_t recent_from)
{
    if (pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The LDS operations of a wavefront are in order: its lanes only have to stay together
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// A workgroup of W wavefronts per sequence and head; a wavefront has a run of slots, 64 of them a stripe.  Ranks are kept in LDS, `held` of each
// wavefront's (longer runs are ranked again).  The rank of the last token that stays is found BITS bits at a time: bins are counted in
// LDS, and every wavefront finds the digit from the counts for itself - lane l has the bins of digits B l .. B l + B - 1, digit B l + k
// at place 64 k + l.  Then the counts of each run say where its places and moves go in the lists: all
// integers, in the order of the slots.
// Bound: vector and LDS instructions of the one compute unit that a row has; 64 rows of 8000 - 32000 tokens 45 us.
template <int W>
struct Evict {
    static constexpr int kThreads = W * kWave;
    static constexpr int kBits = W < 16 ? 8 : 11, kBins = 1 << kBits, kPer = kBins / kWave;
    static constexpr int kHeld = 2048; // ranks of each wavefront: at most 35 and 153 KiB a workgroup
    static constexpr unsigned lds(int held) { return (unsigned)((W * held + kKvBinArrays * kBins + 4 * W) * 4); }
};

template <int W>
__global__ __launch_bounds__(Evict<W>::kThreads) void kv_evict_select_kernel(const KvSeq *__restrict__ seqs, int held, KvShape s, KvEvict e)
{
    constexpr int kBits = Evict<W>::kBits, kBins = Evict<W>::kBins, kPer = Evict<W>::kPer;
    extern __shared__ uint32_t lds[];
    const int wave = wave_number(), lane = threadIdx.x % kWave, row = blockIdx.x;
    uint32_t *bins = lds, *counts = bins + kKvBinArrays * kBins, *ranks = counts + 4 * W + wave * held;
    const KvSeq q = seqs[row / s.n_kv];
    const int head = row % s.n_kv;
    const int64_t at = ((int64_t)q.seq * s.n_kv + head) * s.max_tokens;
    const float *w = e.w_in + at;
    const int32_t *pos = e.pos_in + at;
    const bool copies = e.w_out != e.w_in || e.pos_out != e.pos_in;
    if (q.keep >= q.len) {
        for (int i = wave * kWave + lane; copies && i < q.len; i += W * kWave) {
            e.w_out[at + i] = w[i];
            e.pos_out[at + i] = pos[i];
        }
        return;
    }
    if (q.keep == 0) return;
    const int recent_from = q.seen - min(min(e.recent, q.keep), q.seen);
    const int run = ((q.len + W - 1) / W + kWave - 1) / kWave * kWave;
    const int lo = wave * run, n = max(min(run, q.len - lo), 0); // slots [lo, lo + n)
    // calls f(slot, rank, whether there is such a slot) for the stripes in turn; the lanes stay together
    auto walk = [&](auto f) {
        const int some = min(n, held);
        constexpr int kAhead = 4;
        for (int j0 = 0; j0 < some; j0 += kAhead * kWave) {
            uint32_t r[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) r[k] = ranks[min(j0 + k * kWave, held - kWave) + lane];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int j = j0 + k * kWave;
                if (j < some) f(lo + j + lane, r[k], j + lane < n);
            }
        }
        for (int j = held; j < n; j += kWave) {
            const bool in = j + lane < n;
            f(lo + j + lane, in ? rank_of(w[lo + j + lane], pos[lo + j + lane], recent_from) : 0, in);
        }
    };
    auto place = [](uint32_t digit) { return (digit % kPer) * kWave + digit / kPer; };
    auto count = [&](uint32_t *now, uint32_t digit, bool yes) { // many lanes of one digit: one of them for all
        const uint64_t live = __ballot(yes);
        if (live == 0) return;
        const uint32_t d0 = (uint32_t)__builtin_amdgcn_readlane((int)digit, (int)__ffsll((unsigned long long)live) - 1);
        const uint64_t same = __ballot(yes && digit == d0);
        if (same == live) {
            if (lane == 0) atomicAdd(&now[place(d0)], (uint32_t)__popcll(live));
        } else if (yes) {
            atomicAdd(&now[place(digit)], 1u);
        }
    };

    for (int k = wave * kWave + lane; k < kBins; k += W * kWave) bins[k] = 0;
    __syncthreads();
    // ranks, and the counts of their first bits; eight stripes are loaded together
    constexpr int kAhead = 8;
    for (int j = 0; j < n; j += kAhead * kWave) {
        float a[kAhead];
        int32_t p[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = min(j + k * kWave + lane, n - 1) + lo;
            a[k] = w[i];
            p[k] = pos[i];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = j + k * kWave + lane;
            const uint32_t r = rank_of(a[k], p[k], recent_from);
            if (i - lane < held && i - lane < n) ranks[i] = r;
            const uint32_t digit = r >> (32 - kBits), d0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
            if (__ballot(digit != d0) == 0) { // (recent tokens, tokens that drew nothing; lanes behind the last slot have the last one's)
                if (lane == 0) atomicAdd(&bins[place(d0)], (uint32_t)max(min(n - (i - lane), kWave), 0));
            } else if (i < n) {
                atomicAdd(&bins[place(digit)], 1u);
            }
            if (copies && i < n && lo + i < q.keep) { // (places that fall free are written again, by what moves there)
                e.w_out[at + lo + i] = a[k];
                e.pos_out[at + lo + i] = p[k];
            }
        }
    }
    // the rank of the keep-th token, and how many of that rank stay
    uint32_t prefix = 0;
    int left = q.keep;
    int array = 0;
#pragma unroll 1
    for (int top = 32; top > 0; top -= kBits, array = kv_next_bins(array)) {
        const int shift = max(top - kBits, 0);
        uint32_t *now = bins + array * kBins, *next = bins + kv_next_bins(array) * kBins;
        if (top < 32) {
            const uint32_t mask = (1u << (top - shift)) - 1;
            walk([&](int, uint32_t r, bool in) { count(now, (r >> shift) & mask, in && (r >> top) == (prefix >> top)); });
        }
        if (shift > 0)
            for (int k = wave * kWave + lane; k < kBins; k += W * kWave) next[k] = 0;
        __syncthreads();
        uint32_t c[kPer], mine = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) mine += c[k] = now[k * kWave + lane];
        uint32_t from = mine; // what this lane and those above it count
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) {
            const uint32_t other = (uint32_t)__shfl_down((int)from, x, kWave);
            if (lane + x < kWave) from += other;
        }
        uint32_t above = from - mine;
        const int owner = 63 - (int)__clzll((long long)__ballot(from >= (uint32_t)left)); // the highest lane with enough
        int found = kPer - 1;
#pragma unroll
        for (int k = kPer - 1; k > 0; --k) {
            if (found == k && above + c[k] < (uint32_t)left) {
                above += c[k];
                found = k - 1;
            }
        }
        prefix |= (uint32_t)__builtin_amdgcn_readlane(kPer * lane + found, owner) << shift;
        left -= __builtin_amdgcn_readlane((int)above, owner);
        uint32_t there = c[0];
#pragma unroll
        for (int k = 1; k < kPer; ++k) there = found == k ? c[k] : there;
        if (shift > 0 && prefix > 0 && __builtin_amdgcn_readlane((int)there, owner) == left) { // all of this digit stay: everything above prefix - 1
            prefix -= 1;
            left = 0;
            break;
        }
    }

    // where this run's places and moves go: from what the runs before it have, tokens of greater and of equal rank before and from keep on
    int seen = 0, holes = 0, moves = 0, total = 0; // equal ranks, places, moves so far; all moves
    int c[4] = {0, 0, 0, 0}; // greater and equal before keep, then from keep on
    walk([&](int i, uint32_t r, bool in) {
        const int g = in && r > prefix, same = in && r == prefix, before = i < q.keep;
        c[0] += g & before;
        c[1] += same & before;
        c[2] += g & ~before;
        c[3] += same & ~before;
    });
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int x = 32; x; x >>= 1) c[k] += __shfl_xor(c[k], x, kWave);
        if (lane == 0) counts[k * W + wave] = (uint32_t)c[k];
    }
    __syncthreads();
    int all_seen = 0, all_holes = 0;
    for (int k = 0; k < W; ++k) {
        if (k == wave) seen = all_seen, holes = all_holes, moves = total;
        const int e0 = (int)counts[W + k], e1 = (int)counts[3 * W + k];
        const int stay0 = max(min(left - all_seen, e0), 0), stay1 = max(min(left - all_seen - e0, e1), 0);
        all_holes += max(min(q.keep - k * run, min(run, q.len - k * run)), 0) - (int)counts[k] - stay0;
        total += (int)counts[2 * W + k] + stay1;
        all_seen += e0 + e1;
    }
    const uint64_t lower = (uint64_t(1) << lane) - 1;
    const int most = min(q.keep, q.len - q.keep), blocks = (q.keep + s.N - 1) / s.N;
    int32_t *src = e.src + q.move0 + (int64_t)head * most, *dst = e.dst + q.move0 + (int64_t)head * most;
    int32_t *first = e.first + q.first0 + (int64_t)head * (blocks + 2);
    walk([&](int i, uint32_t r, bool in) {
        const uint64_t same = __ballot(in && r == prefix);
        const bool stays = in && (r > prefix || (r == prefix && seen + (int)__popcll(same & lower) < left));
        seen += (int)__popcll(same);
        if (i - lane < q.keep) { // (a stripe about keep has both)
            const bool hole = in && i < q.keep && !stays;
            const uint64_t hs = __ballot(hole);
            const int h = holes + (int)__popcll(hs & lower);
            if (in && i < q.keep && i % kKvGranule == 0) {
                const int b = (int)kv_div((uint32_t)i / kKvGranule, s.div_b);
                if (b * s.N == i) first[b] = h;
            }
            if (hole) dst[h] = i;
            holes += (int)__popcll(hs);
        }
        const bool move = i >= q.keep && stays;
        const uint64_t ms = __ballot(move);
        if (move) {
            const int m = moves + (int)__popcll(ms & lower);
            src[m] = i;
        }
        moves += (int)__popcll(ms);
    });
    if (wave == 0 && lane == 0) {
        first[blocks] = total;
        // the exponents of the block about the budget, from which tokens move and into which tokens move
        first[blocks + 1] = reinterpret_cast<const int16_t *>(s.exps)[table_entry(s, q.seq, q.keep / s.N, head)];
    }
    __syncthreads();
    // (entries of slots from keep on are only read)
    for (int m = wave * kWave + lane; m < total; m += W * kWave) {
        e.w_out[at + dst[m]] = w[src[m]];
        e.pos_out[at + dst[m]] = pos[src[m]];
    }
}

// A cache at its budget, which has few tokens more than it keeps after each step: a wavefront per row, in one launch.  The token that goes is the one of
// least rank, of equal ones that in the highest slot; the next one is the least behind it in this order.  What stays of
// the slots behind the budget moves at once.
// 64 sequences x 32 heads of 1025 tokens 13 us, 34 MB of weights and positions read and written; kv_evict_select_kernel and kv_evict_move_kernel took 36.
// Bound: the latency of a pass over the row by one wavefront and then of the move.
constexpr int kEvictFew = 4;
__global__ __launch_bounds__(256) void kv_evict_few_kernel(const KvSeq *__restrict__ seqs, int n_rows, KvShape s, KvEvict e)
{
    const int row = blockIdx.x * 4 + wave_number(), lane = threadIdx.x % kWave, D = s.D;
    if (row >= n_rows) return;
    const KvSeq q = seqs[row / s.n_kv];
    const int head = row % s.n_kv;
    const int64_t at = ((int64_t)q.seq * s.n_kv + head) * s.max_tokens;
    const float *w = e.w_in + at;
    const int32_t *pos = e.pos_in + at;
    float *const w_out = e.w_out + at;
    int32_t *const pos_out = e.pos_out + at;
    const bool copies = e.w_out != e.w_in || e.pos_out != e.pos_in;
    const int going = q.keep == 0 ? 0 : q.len - q.keep; // (of none that stay nothing is written)
    if (q.keep == 0 && q.len > 0) return;
    const int recent_from = q.seen - min(min(e.recent, q.keep), q.seen);
    int gone[kEvictFew]; // slots, in the order found
    uint32_t last_rank = 0;
    int last_slot = INT32_MAX;
    for (int turn = 0; turn < max(going, 1); ++turn) {
        uint32_t least = 0xffffffffu;
        int slot = -1;
        constexpr int kAhead = 8;
        for (uint32_t j = 0; j < (uint32_t)q.len; j += kAhead * kWave) {
            float a[kAhead];
            int32_t p[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const uint32_t i = min(j + k * kWave + lane, (uint32_t)q.len - 1);
                a[k] = w[i];
                p[k] = pos[i];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const uint32_t i = j + k * kWave + lane;
                if (turn == 0 && copies && i < (uint32_t)q.keep) { // (places that fall free are written again, by what moves there)
                    w_out[i] = a[k];
                    pos_out[i] = p[k];
                }
                const uint32_t r = rank_of(a[k], p[k], recent_from);
                const bool behind = r > last_rank || (r == last_rank && (int)i < last_slot);
                if (i < (uint32_t)q.len && behind && r <= least) { // (later slots of an equal rank take the place of earlier ones)
                    least = r;
                    slot = (int)i;
                }
            }
        }
        if (going == 0) return;
#pragma unroll
        for (int x = 32; x; x >>= 1) {
            const uint32_t r = (uint32_t)__shfl_xor((int)least, x, kWave);
            const int i = __shfl_xor(slot, x, kWave);
            if (i >= 0 && (slot < 0 || r < least || (r == least && i > slot))) least = r, slot = i;
        }
        slot = __builtin_amdgcn_readfirstlane(slot);
        last_rank = (uint32_t)__builtin_amdgcn_readfirstlane((int)least);
        last_slot = slot;
#pragma unroll
        for (int k = 0; k < kEvictFew; ++k)
            if (k == turn) gone[k] = slot;
    }
    // places and moves, both in the order of the slots: lane k has the k-th slot behind the budget, and the k-th that goes
    __shared__ int moves[4][kEvictFew][2];
    auto &move = moves[wave_number()];
    int mine = INT32_MAX;
#pragma unroll
    for (int k = 0; k < kEvictFew; ++k)
        if (k == lane && k < going) mine = gone[k];
    bool stays = lane < going;
#pragma unroll
    for (int k = 0; k < kEvictFew; ++k) stays = stays && !(k < going && gone[k] == q.keep + lane);
    const uint64_t staying = __ballot(stays);
    int place = 0;
#pragma unroll
    for (int k = 0; k < kEvictFew; ++k) place += k < going && gone[k] < mine;
    const int n = (int)__popcll(staying); // as many places are before the budget
    if (stays) move[__popcll(staying & ((uint64_t(1) << lane) - 1))][0] = q.keep + lane;
    if (mine < q.keep) move[place][1] = mine;
    wave_sync();
    if (lane < n) {
        w_out[move[lane][1]] = w[move[lane][0]];
        pos_out[move[lane][1]] = pos[move[lane][0]];
    }
    const int granule_bytes = 2 * kKvGranule * D;
    auto granule = [&](int64_t entry, int t) { return s.pool + (int64_t)s.table[entry] * s.page_bytes + (int64_t)(t / kKvGranule) * granule_bytes; };
    // a block at a time: all of its moves, since its exponent is that of all
    for (int m0 = 0, m1; m0 < n; m0 = m1) {
        const int block = move[m0][1] / s.N;
        const int64_t entry = table_entry(s, q.seq, block, head);
        const int was_k = s.exps[2 * entry], was_v = s.exps[2 * entry + 1];
        int now_k = was_k, now_v = was_v;
        for (m1 = m0; m1 < n && move[m1][1] / s.N == block; ++m1) {
            const int64_t from = table_entry(s, q.seq, move[m1][0] / s.N, head);
            now_k = max(now_k, (int)s.exps[2 * from]);
            now_v = max(now_v, (int)s.exps[2 * from + 1]);
        }
        const int last = min(s.N, q.keep - block * s.N); // slots of the block that stay in use
        // exponents of sources as they are before this block's change (a block about the budget has places and sources)
        uint32_t k4[kEvictFew];
        uint8_t v1[kEvictFew][4];
        float fk[kEvictFew], fv[kEvictFew];
#pragma unroll
        for (int k = 0; k < kEvictFew; ++k) {
            if (m0 + k >= m1) break;
            const int from = move[m0 + k][0], t = from % s.N;
            const int64_t e0 = table_entry(s, q.seq, from / s.N, head);
            fk[k] = shift_factor(s.exps[2 * e0], now_k);
            fv[k] = shift_factor(s.exps[2 * e0 + 1], now_v);
            const uint8_t *g = granule(e0, t);
            if (lane < D / 4) k4[k] = *(reinterpret_cast<const uint32_t *>(g + t % kKvGranule * D) + lane);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (lane + x * kWave < D) v1[k][x] = g[kKvGranule * D + (lane + x * kWave) * kKvGranule + t % kKvGranule];
        }
        if (now_k != was_k || now_v != was_v) {
            const float grow_k = shift_factor(was_k, now_k), grow_v = shift_factor(was_v, now_v);
            const int words = D / 4;
            for (int u = lane; u < last * words; u += kWave) {
                uint32_t *p = reinterpret_cast<uint32_t *>(granule(entry, u / words) + u / words % kKvGranule * D) + u % words;
                *p = shift_codes(*p, grow_k);
            }
            for (int u = lane; u < (last + 3) / 4 * D; u += kWave) { // four slots of an element
                const int t = u / D * 4;
                uint32_t *p = reinterpret_cast<uint32_t *>(granule(entry, t) + kKvGranule * D + u % D * kKvGranule + t % kKvGranule);
                const uint32_t old = *p, mask = t + 4 <= last ? 0xffffffffu : (1u << (8 * (last - t))) - 1;
                *p = (shift_codes(old, grow_v) & mask) | (old & ~mask); // (the row is this wavefront's alone)
            }
            wave_sync(); // the moved tokens' bytes go over these
        }
#pragma unroll
        for (int k = 0; k < kEvictFew; ++k) {
            if (m0 + k >= m1) break;
            const int t = move[m0 + k][1] - block * s.N;
            uint8_t *g = granule(entry, t);
            if (lane < D / 4) *(reinterpret_cast<uint32_t *>(g + t % kKvGranule * D) + lane) = shift_codes(k4[k], fk[k]);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (lane + x * kWave < D) g[kKvGranule * D + (lane + x * kWave) * kKvGranule + t % kKvGranule] = (uint8_t)shift_codes(v1[k][x], fv[k]);
        }
        if (lane < 2) s.exps[2 * entry + lane] = (int8_t)(lane ? now_v : now_k);
    }
}

// A workgroup = some of the blocks of a row (sequence and head) that keep tokens, those that take any.  Nobody writes slots from keep on,
// and nobody else these blocks'.  A thread has 16 bytes of a token's K, or the eight tokens of a granule in one element
// of V: what stays (shifted, if a larger exponent comes) and what comes are put together in registers.
// Bound: V's bytes, a line of which holds 16 elements of eight tokens; 64 rows that take about 1900 tokens each 34 us.
constexpr int kMoveThreads = 256;
__global__ __launch_bounds__(kMoveThreads) void kv_evict_move_kernel(const KvSeq *__restrict__ seqs, KvShape s, KvEvict e)
{
    // of each slot of the block (a page holds at most 32768 / 32 tokens): where its token comes from, as the address of element 0 of K; V's
    // is behind.  Its own place, if it stays.
    __shared__ const uint8_t *from_k[1024], *from_v[1024];
    __shared__ float factor[2][1024];
    __shared__ __align__(8) uint8_t comes[1024];
    const KvSeq q = seqs[blockIdx.x / s.n_kv];
    if (q.keep >= q.len) return;
    const int head = blockIdx.x % s.n_kv, D = s.D, lane = threadIdx.x % kWave;
    const int blocks = (q.keep + s.N - 1) / s.N;
    const int most = min(q.keep, q.len - q.keep);
    const int32_t *src = e.src + q.move0 + (int64_t)head * most, *dst = e.dst + q.move0 + (int64_t)head * most;
    const int32_t *first = e.first + q.first0 + (int64_t)head * (blocks + 2);
    // exponents of a source, K's in the low byte: of blocks behind the budget, which nobody changes, or as the block about it had them
    auto exponents_of = [&](int slot) {
        const int b = (int)kv_div((uint32_t)slot / kKvGranule, s.div_b);
        return b == q.keep / s.N ? first[blocks + 1] : (int)reinterpret_cast<const int16_t *>(s.exps)[table_entry(s, q.seq, b, head)];
    };
    const int granule_bytes = 2 * kKvGranule * D;
    // blocks y, y + gridDim.y, ...: 64 at a time
    for (int k0 = 0; (int)blockIdx.y + k0 * (int)gridDim.y < blocks; k0 += kWave) {
        const int mine = (int)blockIdx.y + (k0 + lane) * (int)gridDim.y;
        uint64_t busy = __ballot(mine < blocks && first[mine] < first[mine + 1]);
        while (busy) {
            const int block = (int)blockIdx.y + (k0 + (int)__ffsll((unsigned long long)busy) - 1) * (int)gridDim.y;
            busy &= busy - 1;
            const int m0 = first[block], m1 = first[block + 1];
            const int64_t entry = table_entry(s, q.seq, block, head);
            uint8_t *page = s.pool + (int64_t)s.table[entry] * s.page_bytes;
            const int was_k = s.exps[2 * entry], was_v = s.exps[2 * entry + 1];
            int now_k = was_k, now_v = was_v;
            for (int m = m0 + lane; m < m1; m += kWave) {
                const int both = exponents_of(src[m]);
                now_k = max(now_k, (int)(int8_t)(both & 0xff));
                now_v = max(now_v, both >> 8);
            }
#pragma unroll
            for (int x = 32; x; x >>= 1) {
                now_k = max(now_k, __shfl_xor(now_k, x, kWave));
                now_v = max(now_v, __shfl_xor(now_v, x, kWave));
            }
            const int last = min(s.N, q.keep - block * s.N); // slots of the block that stay in use
            auto granule = [&](const uint8_t *base, int t) { return base + (int64_t)(t / kKvGranule) * granule_bytes; };
            __syncthreads(); // the block before is done
            for (int t = threadIdx.x; t < s.N; t += kMoveThreads) {
                from_k[t] = granule(page, t) + (t % kKvGranule) * D;
                from_v[t] = granule(page, t) + kKvGranule * D + t % kKvGranule;
                factor[0][t] = shift_factor(was_k, now_k);
                factor[1][t] = shift_factor(was_v, now_v);
                comes[t] = 0;
            }
            __syncthreads();
            for (int m = m0 + (int)threadIdx.x; m < m1; m += kMoveThreads) {
                const int t = dst[m] - block * s.N, from = src[m], r = from % s.N, both = exponents_of(from);
                const uint8_t *there = granule(s.pool + (int64_t)s.table[table_entry(s, q.seq, from / s.N, head)] * s.page_bytes, r);
                from_k[t] = there + (r % kKvGranule) * D;
                from_v[t] = there + kKvGranule * D + r % kKvGranule;
                factor[0][t] = shift_factor((int8_t)(both & 0xff), now_k);
                factor[1][t] = shift_factor(both >> 8, now_v);
                comes[t] = 1;
            }
            __syncthreads();
            const int chunks = D / 16;
            for (int u = threadIdx.x; u < last * chunks; u += kMoveThreads) {
                const int t = u / chunks;
                if (!comes[t] && now_k == was_k) continue;
                const u32x4 c = *(reinterpret_cast<const u32x4 *>(from_k[t]) + u % chunks);
                u32x4 r;
#pragma unroll
                for (int k = 0; k < 4; ++k) r[k] = shift_codes(c[k], factor[0][t]);
                *(reinterpret_cast<u32x4 *>(page + (int64_t)(t / kKvGranule) * granule_bytes + (t % kKvGranule) * D) + u % chunks) = r;
            }
            for (int u = threadIdx.x; u < (last + kKvGranule - 1) / kKvGranule * D; u += kMoveThreads) {
                const int g = u / D, d = u % D, t0 = g * kKvGranule;
                if (*reinterpret_cast<const uint64_t *>(&comes[t0]) == 0 && now_v == was_v) continue;
                uint32_t c[kKvGranule];
#pragma unroll
                for (int t = 0; t < kKvGranule; ++t) c[t] = from_v[t0 + t][d * kKvGranule];
                uint32_t r[2] = {0, 0};
#pragma unroll
                for (int t = 0; t < kKvGranule; ++t)
                    r[t / 4] |= ((uint32_t)(int)__builtin_rintf((float)(int8_t)c[t] * factor[1][t0 + t]) & 0xffu) << (8 * (t % 4));
                uint8_t *to = page + (int64_t)g * granule_bytes + kKvGranule * D + d * kKvGranule;
                if (t0 + kKvGranule <= last) {
                    *reinterpret_cast<u32x2 *>(to) = u32x2{r[0], r[1]};
                } else { // others may be reading the slots behind
                    for (int t = 0; t0 + t < last; ++t) to[t] = (uint8_t)(r[t / 4] >> (8 * (t % 4)));
                }
            }
            if (threadIdx.x == 0) { // (everyone has read them: two barriers ago)
                s.exps[2 * entry] = (int8_t)now_k;
                s.exps[2 * entry + 1] = (int8_t)now_v;
            }
        }
    }
}

// f(integral constants of the type and of D / 32)
template <typename F>
int32_t by_shape(int dtype, int D, F f)
{
    auto of = [&](auto dt) -> int32_t {
        switch (D / 32) {
        case 1: return f(dt, std::integral_constant<int, 1>{});
        case 2: return f(dt, std::integral_constant<int, 2>{});
        case 3: return f(dt, std::integral_constant<int, 3>{});
        case 4: return f(dt, std::integral_constant<int, 4>{});
        case 6: return f(dt, std::integral_constant<int, 6>{});
        case 8: return f(dt, std::integral_constant<int, 8>{});
        }
        return fail(SLORA_EINVAL, "no kernel for head_dim=%d", D);
    };
    return dtype == SLORA_F16 ? of(std::integral_constant<int, SLORA_F16>{}) : of(std::integral_constant<int, SLORA_BF16>{});
}

} // namespace

int32_t launch_kv_table(const slora_kv8_batch *b, void *stream)
{
    hipLaunchKernelGGL(kv_table_kernel, dim3((unsigned)b->columns.size()), dim3(256), 0, (hipStream_t)stream, b->cache->d_table, b->d_columns, b->d_pages,
                       b->cache->per_block());
    return check_launch("kv_table");
}

int32_t launch_kv_append(const slora_kv8_batch *b, const KvShape &shape, const KvAppend &a, void *stream)
{
    if (b->append.empty()) return SLORA_OK;
    const dim3 grid((unsigned)(b->append.size() * shape.n_kv)), block(2 * kWave);
    if (b->cache->pool->dtype == SLORA_F16)
        hipLaunchKernelGGL(kv_append_kernel<SLORA_F16>, grid, block, 0, (hipStream_t)stream, b->d_append, b->d_seqs, shape, a);
    else
        hipLaunchKernelGGL(kv_append_kernel<SLORA_BF16>, grid, block, 0, (hipStream_t)stream, b->d_append, b->d_seqs, shape, a);
    return check_launch("kv_append");
}

// Parts of a column, up to which a wavefront puts them together alone.  us a pass, by a wavefront / by four: two sequences of 90000 - 131000 tokens (64 parts) 96 / 84, 32 of nine
// drafted tokens behind 2000 (8 heads) 78 / 85, 64 of 500 - 8000 124 / 126.
constexpr int32_t kFewParts = 16;

int32_t launch_kv_attend(const slora_kv8_batch *b, const KvShape &shape, const KvAttend &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    return by_shape(b->cache->pool->dtype, shape.D, [&](auto dt, auto db) {
        int32_t rc = SLORA_OK;
        if (!b->many.empty()) { // (the longer ones)
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_attend_many_kernel<dt.value, db.value>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
            if (e != hipSuccess) return fail(SLORA_EHIP, "hipFuncSetAttribute(LDS size): %s", hipGetErrorString(e));
            hipLaunchKernelGGL((kv_attend_many_kernel<dt.value, db.value>), dim3((unsigned)(b->many.size() * shape.n_kv)), dim3(kKvManyThreads),
                               sizeof(ManyLds<db.value>), st, b->d_many, b->d_seqs, shape, a);
            rc = check_launch("kv_attend_many");
        }
        if (rc == SLORA_OK && !b->few.empty()) {
            hipLaunchKernelGGL((kv_attend_few_kernel<dt.value, db.value>), dim3((unsigned)(b->few.size() * shape.n_kv)), dim3(kKvFewThreads), 0, st, b->d_few,
                               b->d_seqs, shape, a);
            rc = check_launch("kv_attend_few");
        }
        if (rc == SLORA_OK && !b->join.empty()) {
            const unsigned items = (unsigned)(b->join.size() * shape.n_kv);
            if (b->join_parts > kFewParts)
                hipLaunchKernelGGL((kv_join_kernel<dt.value, db.value, 4>), dim3(items, (unsigned)b->join_cols), dim3(256), 0, st, b->d_join, b->d_seqs, shape, a);
            else
                hipLaunchKernelGGL((kv_join_kernel<dt.value, db.value, 1>), dim3(items, (unsigned)(b->join_cols + 3) / 4), dim3(256), 0, st, b->d_join, b->d_seqs,
                                   shape, a);
            rc = check_launch("kv_join");
        }
        return rc;
    });
}

int32_t launch_kv_weights(const slora_kv8_batch *b, const KvShape &shape, const KvAttend &a, const KvWeights &w, void *stream)
{
    if (b->longest == 0) return SLORA_OK;
    if (b->longest_few > 0) {
        const dim3 grid((unsigned)((b->longest_few + 255) / 256), (unsigned)shape.n_kv, (unsigned)b->seqs.size());
        hipLaunchKernelGGL(kv_weights_few_kernel, grid, dim3(256), 0, (hipStream_t)stream, b->d_seqs, shape, a, w);
        int32_t rc = check_launch("kv_weights_few");
        if (rc != SLORA_OK || b->longest_many == 0) return rc;
    }
    const dim3 grid((unsigned)((b->longest_many + 127) / 128), (unsigned)shape.n_kv, (unsigned)b->seqs.size());
    return by_shape(b->cache->pool->dtype, shape.D, [&](auto dt, auto db) {
        hipLaunchKernelGGL((kv_weights_kernel<dt.value, db.value>), grid, dim3(256), 0, (hipStream_t)stream, b->d_seqs, shape, a, w);
        return check_launch("kv_weights");
    });
}

int32_t launch_kv_evict(const slora_kv8_batch *b, const KvShape &shape, const KvEvict &e, void *stream)
{
    const int64_t rows = (int64_t)b->seqs.size() * shape.n_kv;
    hipStream_t st = (hipStream_t)stream;
    // A wavefront reads a row again for every token that goes.  us, it / the other kernels: 2048 rows of 1025 tokens, one goes 13 / 39, of 8000, four go 129 / 144,
    // of 16000, one goes 113 / 313; 512 rows of 8000, two go 48 / 52, of 16000, one goes 58 / 85; 256 rows of 8000, two go 47 / 33; 32 rows of 8000, one goes 24 / 31,
    // four go 79 / 31, of 32000, one goes 83 / 60; 128 rows of 4000, two go 25 / 27.
    if (b->most_going <= kEvictFew && (int64_t)std::max(b->most_going, 1) * b->longest <= (rows >= 512 ? 32768 : 8192)) {
        hipLaunchKernelGGL(kv_evict_few_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, b->d_seqs, (int)rows, shape, e);
        return check_launch("kv_evict_few");
    }
    auto select = [&](auto w) -> int32_t {
        typedef Evict<w.value> E;
        // stripes of the longest run, at most what LDS holds
        const int held = std::min<int>(E::kHeld, ((b->longest + w.value - 1) / w.value + kWave - 1) / kWave * kWave);
        if (E::lds(held) > 65536) {
            const hipError_t a = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_evict_select_kernel<w.value>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
            if (a != hipSuccess) return fail(SLORA_EHIP, "hipFuncSetAttribute(LDS size): %s", hipGetErrorString(a));
        }
        hipLaunchKernelGGL(kv_evict_select_kernel<w.value>, dim3((unsigned)rows), dim3(E::kThreads), E::lds(held), st,
                           b->d_seqs, held, shape, e);
        return check_launch("kv_evict_select");
    };
    // us with 4 / 16 wavefronts: 2048 rows of 1025 tokens 101 / 189, of 8000 450 / 524, 512 of 8000 121 / 125, of 16000 745 / 649; where a row has a compute unit for
    // itself, 256 rows of 5000 65 / 60, of 8000 78 / 65, 128 of 2000 35 / 39, of 4000 45 / 43, of 8000 61 / 48, of 30000 478 / 241.  (One wavefront: 2048 rows of 1025 99,
    // of 2040 181 where four take 167.)
    const bool wide = b->longest > (rows > 256 ? 8192 : 4096);
    int32_t rc = wide ? select(std::integral_constant<int, 16>{}) : select(std::integral_constant<int, 4>{});
    if (rc == SLORA_OK && b->dest_blocks > 0) {
        // eight workgroups for every compute unit
        const int64_t split = std::max<int64_t>(1, std::min<int64_t>(b->dest_blocks, (2048 + rows - 1) / rows));
        hipLaunchKernelGGL(kv_evict_move_kernel, dim3((unsigned)rows, (unsigned)split), dim3(kMoveThreads), 0, st, b->d_seqs, shape, e);
        rc = check_launch("kv_evict_move");
    }
    return rc;
}

} // namespace slora
