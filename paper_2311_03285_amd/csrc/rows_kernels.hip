// gfx950 kernels on whole rows: norms around a block with its gate and residual, rows in 8 bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "rows.hpp"

namespace slora {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------
// a row in registers
// ---------------------------------------------------------------------------------------
// A row belongs to `waves` wavefronts and stays in their registers from its one load to its stores.  Its pieces of eight elements are dealt out in
// turn, P to a lane at most; a last piece that is not whole (TAIL) is read as the 16-byte words that it begins in, and
// written element by element, so that nothing behind the row is touched.  (Read by elements it cost norms of 777 rows of 5003 elements 3 of 21 us.)
// Loads are not behind branches: a lane without a piece reads the row's last one once more.
template <int P, bool TAIL>
struct Row {
    int lane, lanes; // of the row
    int width, pieces;
    __device__ __forceinline__ int piece(int p) const { return lane + p * lanes; }
    __device__ __forceinline__ bool has(int p) const { return piece(p) < pieces; }
    __device__ __forceinline__ bool whole(int p) const { return !TAIL || (piece(p) + 1) * kPiece <= width; } // of one that there is
    __device__ __forceinline__ bool valid(int p, int i) const { return TAIL ? piece(p) * kPiece + i < width : has(p); }
    __device__ __forceinline__ int at(int p) const { return min(piece(p), pieces - 1) * kPiece; }
    __device__ __forceinline__ int count(int wave) const // elements of a wavefront
    {
        int n = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) n += min(max(width - (p * lanes + wave * kWave) * kPiece, 0), kWave * kPiece);
        return n;
    }
};

// The same row for a next pass, whose comparisons are made anew: kept from pass to pass they take more scalar registers than there are.
template <int P, bool TAIL>
__device__ __forceinline__ Row<P, TAIL> again(Row<P, TAIL> r)
{
    if constexpr (TAIL) asm volatile("" : "+v"(r.lane));
    return r;
}

template <int DT>
__device__ __forceinline__ void widen8(const u32x4 &raw, float (&v)[kPiece])
{
#pragma unroll
    for (int i = 0; i < kPiece; ++i) v[i] = widen<DT>((uint16_t)(raw[i / 2] >> (16 * (i % 2))));
}

// ONCE: rows are loaded without a place in the caches (vectors that all rows read always with one): those of calls with this many bytes of them or more.  No bound of a cache: the
// memory-side one holds 256 MiB and may have rows of this size from the kernel that wrote them; by what was measured.  us with / without a place, rows that a product has just written:
// gated products of 2048 rows of 20480 (160 MiB) 54.8 / 53.7, 3000 (234) 80.6 / 73.9, 1024 (80) 28.9 / 25.6, a norm of 8192 rows of 5120 (160) 63.0 / 57.9, of 4096 (80) 32.3 / 35.2;
// rows that are in no cache: 4096 of 5120 (40) 13.5 / 13.6, 2048 of 20480 (80) 29.6 / 30.3, norms of 8192 of 4096 48.7 / 44.5; rows read again from the memory-side cache: 4096 of
// 5120 12.1 / 12.6, 2048 of 20480 25.0 / 30.4.
constexpr int64_t kOnceBytes = 64 << 20;
template <bool ONCE, typename T>
__device__ __forceinline__ T load_piece(const T *from)
{
    if constexpr (ONCE)
        return __builtin_nontemporal_load(from);
    else
        return *from;
}

// a 16-bit vector's pieces as they are
template <bool ONCE, int P, bool TAIL>
__device__ __forceinline__ void load16(const Row<P, TAIL> &r, const uint16_t *from, u32x4 (&raw)[P])
{
#pragma unroll
    for (int p = 0; p < P; ++p) raw[p] = load_piece<ONCE>(reinterpret_cast<const u32x4 *>(from + r.at(p)));
}
template <bool ONCE, int P, bool TAIL>
__device__ __forceinline__ void load32(const Row<P, TAIL> &r, const float *from, f32x4 (&raw)[P][2])
{
#pragma unroll
    for (int p = 0; p < P; ++p) {
        raw[p][0] = load_piece<ONCE>(reinterpret_cast<const f32x4 *>(from + r.at(p)));
        raw[p][1] = load_piece<ONCE>(reinterpret_cast<const f32x4 *>(from + (TAIL ? min(r.at(p) + 4, (r.width - 1) / 4 * 4) : r.at(p) + 4)));
    }
}
template <int DT, int P, bool TAIL>
__device__ __forceinline__ void store16(const Row<P, TAIL> &row, uint16_t *to, const float (&v)[P][kPiece])
{
    const Row<P, TAIL> r = again(row);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!r.has(p)) continue;
        uint16_t e[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) e[i] = narrow<DT>(v[p][i]);
        if (r.whole(p)) {
            u32x4 u;
#pragma unroll
            for (int i = 0; i < kPiece / 2; ++i) u[i] = (uint32_t)e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
            *reinterpret_cast<u32x4 *>(to + r.at(p)) = u;
        } else {
#pragma unroll
            for (int i = 0; i < kPiece - 1; ++i)
                if (r.valid(p, i)) to[r.at(p) + i] = e[i];
        }
    }
}
template <int P, bool TAIL>
__device__ __forceinline__ void store32(const Row<P, TAIL> &row, float *to, const float (&v)[P][kPiece])
{
    const Row<P, TAIL> r = again(row);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!r.has(p)) continue;
        if (r.whole(p)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4 *>(to + r.at(p) + 4 * i) = f32x4{v[p][4 * i], v[p][4 * i + 1], v[p][4 * i + 2], v[p][4 * i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < kPiece - 1; ++i)
                if (r.valid(p, i)) to[r.at(p) + i] = v[p][i];
        }
    }
}

// ---------------------------------------------------------------------------------------
// sums and maxima over a row
// ---------------------------------------------------------------------------------------
// over the wavefront, without LDS: lanes of 16 by shifts, then what the 16s before have found; the total is the last lane's
__device__ __forceinline__ float wave_sum(float v)
{
#define SLORA_STEP(control, rows) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), control, rows, 0xf, false))
    SLORA_STEP(0x111, 0xf); // row_shr 1, 2, 4, 8
    SLORA_STEP(0x112, 0xf);
    SLORA_STEP(0x114, 0xf);
    SLORA_STEP(0x118, 0xf);
    SLORA_STEP(0x142, 0xa); // row_bcast 15, 31
    SLORA_STEP(0x143, 0xc);
#undef SLORA_STEP
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
__device__ __forceinline__ int wave_max(int v)
{
#define SLORA_STEP(control) v = max(v, __builtin_amdgcn_update_dpp(v, v, control, 0xf, 0xf, false))
    SLORA_STEP(0x111);
    SLORA_STEP(0x112);
    SLORA_STEP(0x114);
    SLORA_STEP(0x118);
    SLORA_STEP(0x142);
    SLORA_STEP(0x143);
#undef SLORA_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

// Over the row's wavefronts, in their order.  Each reduction has words of its own, so one barrier does.
struct Team {
    uint32_t (*slots)[kRowThreads / kWave];
    int waves, wave, used = 0;
    // every wavefront's v, behind the next barrier
    __device__ __forceinline__ const float *share(float v)
    {
        float *s = reinterpret_cast<float *>(slots[used++]);
        if (threadIdx.x % kWave == 0) s[wave] = v;
        return s;
    }
    __device__ __forceinline__ float sum(float v)
    {
        v = wave_sum(v);
        if (waves == 1) return v;
        const float *const s = share(v);
        __syncthreads();
        v = 0.0f;
        for (int w = 0; w < waves; ++w) v += s[w];
        return v;
    }
    __device__ __forceinline__ int max_of(int v)
    {
        v = wave_max(v);
        if (waves == 1) return v;
        uint32_t *s = slots[used++];
        if (threadIdx.x % kWave == 0) s[wave] = (uint32_t)v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < waves; ++w) v = max(v, (int)s[w]);
        return v;
    }
};
constexpr int kReductions = 11; // most of a row: two norms of five (mean, spread, maximum, mean, spread) and the codes' maximum

// bits of a magnitude: in the order of the numbers, NaN above infinity
__device__ __forceinline__ int magnitude(float v) { return (int)(__float_as_uint(v) & 0x7fffffffu); }

template <int P, bool TAIL>
__device__ __forceinline__ int largest(const Row<P, TAIL> &row, const float (&v)[P][kPiece], Team &team)
{
    const Row<P, TAIL> r = again(row);
    int top = 0;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) top = max(top, r.valid(p, i) ? magnitude(v[p][i]) : 0);
    return team.max_of(top);
}

// ---------------------------------------------------------------------------------------
// norms
// ---------------------------------------------------------------------------------------
struct Spread {
    float mean, square; // square: mean square of v - mean
};
// Layer norms: each wavefront's mean and its sum of squares about that, put together with one barrier: the squares about the row's mean are
// those plus count * (difference of means)^2.  All terms are positive; nothing cancels.
template <int P, bool TAIL>
__device__ __forceinline__ Spread spread_of(const Row<P, TAIL> &row, const float (&v)[P][kPiece], bool layer, int width, Team &team)
{
    Row<P, TAIL> r = again(row);
    Spread s{0.0f, 0.0f};
    if (layer) {
        float sum = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) sum += r.valid(p, i) ? v[p][i] : 0.0f;
        s.mean = wave_sum(sum) / (float)max(r.count(team.waves == 1 ? 0 : team.wave), 1);
        r = again(r);
    }
    float sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float d = r.valid(p, i) ? v[p][i] - s.mean : 0.0f;
            sum = __builtin_fmaf(d, d, sum);
        }
    if (layer && team.waves > 1) {
        const float *const square = team.share(wave_sum(sum)), *const mean = team.share(s.mean);
        __syncthreads();
        float total = 0.0f;
        for (int w = 0; w < team.waves; ++w) total = __builtin_fmaf(mean[w], (float)r.count(w), total);
        s.mean = total / (float)width;
        total = 0.0f;
        for (int w = 0; w < team.waves; ++w) {
            const float d = mean[w] - s.mean;
            total += __builtin_fmaf(d * d, (float)r.count(w), square[w]);
        }
        s.square = total / (float)width;
    } else {
        s.square = team.sum(sum) / (float)width;
    }
    return s;
}

// v = (v - mean) / sqrt(mean square + eps), with all of the row in registers: the spread is of differences, not a difference of sums.
// Squares that leave fp32's range (bfloat16 and fp32 rows can) are taken again of v times a power of two, which is
// exact; eps, which is 0 or at least 2^-60, is scaled along.  With an eps, squares are never too small, and rows are only scaled down; what is left of eps is then far
// below any spread but 0, and must not become 0 itself: a layer norm of equal values is 0, however large they are.  All lanes of the row go the same way.
template <int P, bool TAIL>
__device__ __forceinline__ void normalise(const Row<P, TAIL> &r, float (&v)[P][kPiece], bool layer, int width, float eps, Team &team)
{
    Spread s = spread_of(r, v, layer, width, team);
    float q = s.square + eps;
    if (!(q >= 0x1p-80f && q <= 0x1p100f)) {
        const int top = largest(r, v, team);
        if (top < 0x7f800000) { // (an infinity or NaN spoils its row either way)
            // the largest magnitude to about 1, or (eps) to that at most: factors 2^up, two of them where one is no normal number
            const int up = 127 - max(top >> 23, eps > 0.0f ? 127 : 1);
            const float a = __uint_as_float((uint32_t)(127 + up / 2) << 23), b = __uint_as_float((uint32_t)(127 + (up - up / 2)) << 23);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[p][i] = v[p][i] * a * b;
            s = spread_of(r, v, layer, width, team);
            q = s.square + (eps > 0.0f ? fmaxf(eps * a * b * a * b, 0x1p-126f) : 0.0f);
        }
    }
    const float by = 1.0f / sqrtf(q);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[p][i] = (v[p][i] - s.mean) * by;
}

// v = v * weight + bias, where there are any
template <int DT, int P, bool TAIL>
__device__ __forceinline__ void affine(const Row<P, TAIL> &r, float (&v)[P][kPiece], const u32x4 (&weight)[P], const uint16_t *w,
                                       const uint16_t *bias)
{
    if (w) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float e[kPiece];
            widen8<DT>(weight[p], e);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[p][i] *= e[i];
        }
    }
    if (bias) {
        u32x4 raw[P];
        load16<false>(r, bias, raw);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float e[kPiece];
            widen8<DT>(raw[p], e);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[p][i] += e[i];
        }
    }
}

// ---------------------------------------------------------------------------------------
// 8 bits
// ---------------------------------------------------------------------------------------
// Codes are rounded from fp32 values (not from the 16 bits that x is rounded to: one rounding, not two).
template <int P, bool TAIL>
__device__ __forceinline__ void store_codes(const Row<P, TAIL> &row, const RowsOut &out, int64_t t, const float (&v)[P][kPiece], Team &team)
{
    const int top = largest(row, v, team);
    const Row<P, TAIL> r = again(row);
    const bool spoiled = top >= 0x7f800000;
    const float a = fmaxf(__uint_as_float((uint32_t)top), kW8Least), inverse = spoiled ? 0.0f : 1.0f / a * 127.0f;
    int8_t *to = out.codes + t * out.codes_stride;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!r.has(p)) continue;
        uint32_t c[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) c[i] = spoiled ? 0u : (uint32_t)(int)__builtin_rintf(v[p][i] * inverse) & 0xffu;
        if (r.whole(p)) {
            u32x2 u;
#pragma unroll
            for (int i = 0; i < 2; ++i) u[i] = c[4 * i] | c[4 * i + 1] << 8 | c[4 * i + 2] << 16 | c[4 * i + 3] << 24;
            *reinterpret_cast<u32x2 *>(to + r.at(p)) = u;
        } else {
#pragma unroll
            for (int i = 0; i < kPiece - 1; ++i)
                if (r.valid(p, i)) to[r.at(p) + i] = (int8_t)c[i];
        }
    }
    if (r.lane == 0) out.scales[t] = spoiled ? __uint_as_float(0x7fc00000u) : a / 127.0f;
}

constexpr int kGridX = 1 << 20; // workgroups along x: with 1024 threads each they stay below 2^32 threads

template <int P, bool TAIL>
__device__ __forceinline__ Row<P, TAIL> row_of(int width, int waves)
{
    Row<P, TAIL> r;
    r.lanes = waves * kWave;
    r.lane = waves == 1 ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    r.width = width;
    r.pieces = (width + kPiece - 1) / kPiece;
    return r;
}

__device__ __forceinline__ int64_t row_number(int waves, int wave)
{
    const int64_t block = (int64_t)blockIdx.y * kGridX + blockIdx.x;
    return waves == 1 ? block * (blockDim.x / kWave) + wave : block;
}

// One row for the workgroup, or (waves == 1) one for each of its wavefronts.
// Bound: HBM where there are rows enough (8192 rows of 8192, a norm behind the block and a gate by channel, 537 MB: 97 us = 5.5 TB/s, a copy reaches 5.05; from memory 2048
// of 4096 15.5 us = 4.3 TB/s, 12.6 where they are in the memory-side cache); below, the chain of two loads, two to four reductions and a store (777 rows of 5003 in fp32, gate by token: 19.6 us from
// memory = 2.8 TB/s, 15 in that cache), and the launch (one row 6.1 - 7.5 us, 3.4 in the kernel).
template <int DT, bool H32, int P, bool TAIL, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void norm_kernel(NormArgs a, int waves)
{
    __shared__ uint32_t slots[kReductions][kRowThreads / kWave];
    const int wave = wave_number();
    const int64_t t = row_number(waves, wave);
    if (t >= a.T) return; // (all wavefronts that share barriers)
    const Row<P, TAIL> r = row_of<P, TAIL>(a.width, waves);
    Team team{slots, waves, wave};

    // With four pieces a lane nothing is loaded before it is needed: what is under way early takes registers that more wavefronts can use.  us with / without: 2048
    // rows of 16384 54 / 51, 8192 of 8192 98 / 96, 777 of 5003 20 / 20.
    constexpr bool kAhead = P <= 2;
    auto not_before = [] {
        if constexpr (!kAhead) asm volatile("" ::: "memory");
    };
    float v[P][kPiece];
    typedef typename std::conditional<H32, f32x4[P][2], u32x4[P]>::type Raw;
    Raw h;
    auto load_h = [&] {
        if constexpr (H32)
            load32<ONCE>(r, static_cast<const float *>(a.h) + t * a.h_stride, h);
        else
            load16<ONCE>(r, static_cast<const uint16_t *>(a.h) + t * a.h_stride, h);
    };
    if constexpr (kAhead) load_h();
    if (a.block) {
        u32x4 raw[P], weight[P], gate[P];
        auto load_weight = [&] {
            if (a.post && a.post_weight) load16<false>(r, a.post_weight, weight);
        };
        auto load_gate = [&] {
            if (a.gate && a.gate_stride) load16<ONCE>(r, a.gate + t * a.gate_stride, gate);
            if (a.gate && !a.gate_stride) load16<false>(r, a.gate, gate);
        };
        load16<ONCE>(r, a.block + t * a.block_stride, raw);
        if constexpr (kAhead) load_weight();
        if constexpr (kAhead) load_gate();
#pragma unroll
        for (int p = 0; p < P; ++p) widen8<DT>(raw[p], v[p]);
        if (a.post) {
            normalise(r, v, a.layer != 0, a.width, a.eps, team);
            not_before();
            if constexpr (!kAhead) load_weight();
            affine<DT>(r, v, weight, a.post_weight, a.post_bias);
        }
        not_before();
        if constexpr (!kAhead) load_gate();
        if (a.gate) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float e[kPiece];
                widen8<DT>(gate[p], e);
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[p][i] *= e[i];
            }
        }
    }
    not_before();
    if constexpr (!kAhead) load_h();
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float e[kPiece];
        if constexpr (H32) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) e[i] = h[p][i / 4][i % 4];
        } else {
            widen8<DT>(h[p], e);
        }
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[p][i] = a.block ? __builtin_fmaf(a.scale, v[p][i], e[i]) : e[i];
    }
    if (a.h_out) {
        if constexpr (H32)
            store32(r, static_cast<float *>(a.h_out) + t * a.h_out_stride, v);
        else
            store16<DT>(r, static_cast<uint16_t *>(a.h_out) + t * a.h_out_stride, v);
    }
    if (!a.out.x && !a.out.codes) return;
    u32x4 weight[P];
    auto load_weight = [&] {
        if (a.pre_weight) load16<false>(r, a.pre_weight, weight);
    };
    if constexpr (kAhead) load_weight();
    normalise(r, v, a.layer != 0, a.width, a.eps, team);
    not_before();
    if constexpr (!kAhead) load_weight();
    affine<DT>(r, v, weight, a.pre_weight, a.pre_bias);
    if (a.out.x) store16<DT>(r, a.out.x + t * a.out.x_stride, v);
    if (a.out.codes) store_codes(r, a.out, t, v, team);
}

// x act(g) with act(g) = g / (1 + z), z = exp(-u): u = g, or (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u)) with u = 2 sqrt(2 / pi) (g + 0.044715 g^3).
// z = 2^(n + r) with whole n and |r| <= 1, so that only r is rounded: u log2 e is a product (two with the cube) of a constant in two parts, less its whole part, in
// one fused step.  (u log2 e rounded as a number would be off by |u| half-steps of z.)  2^r and 1 / (1 + z) are the hardware's, good to a step each.  All of it is off
// by at most 12 half-steps of fp32, counted: r's 4 roundings 1.4, the exponential 2, both once more in 1 + z, that sum 1, its reciprocal 2, up to three products.
template <int DT, int ACT>
struct Gate {
    static constexpr double kLog2e = 1.44269504088896340736, kA = ACT == SLORA_ACT_SILU ? kLog2e : 2.0 * 0.79788456080286535588 * kLog2e, kB = 0.044715 * kA;
    static constexpr float kAHigh = (float)kA, kALow = (float)(kA - kAHigh), kBHigh = (float)kB, kBLow = (float)(kB - kBHigh);
    // z = power * 2^whole
    float power;
    int whole;
    __device__ __forceinline__ explicit Gate(float g)
    {
        float n = __builtin_rintf(g * -kAHigh), r = __builtin_fmaf(g, -kALow, __builtin_fmaf(g, -kAHigh, -n));
        if constexpr (ACT == SLORA_ACT_GELU) {
            const float square = g * g, cube = square * g, m = __builtin_rintf(cube * -kBHigh); // (of 16-bit numbers: the square is exact, and of bfloat16 the cube)
            float part = __builtin_fmaf(cube, -kBLow, __builtin_fmaf(cube, -kBHigh, -m));
            if constexpr (DT == SLORA_F16) part = __builtin_fmaf(__builtin_fmaf(square, g, -cube), -kBHigh, part);
            n += m;
            r += part;
        }
        power = __builtin_amdgcn_exp2f(r);
        whole = (int)n;
    }
    __device__ __forceinline__ float z() const { return __builtin_ldexpf(power, whole); }
    static __device__ __forceinline__ float quotient(float z) { return __builtin_amdgcn_rcpf(1.0f + z); }
    // Gates from -kSmall to kSmall: z < 2^96 and its quotient are in range.  silu needs no whole part there: what t = -g log2 e is off by as a number is -g - t ln 2, one fused step, by
    // which z is put right.  (ln 2 is off by 0.05 half-steps, of up to 40: 1.9; the exponential 2, this step 1, 1 + z 1, its reciprocal 2, two products.)
    static constexpr float kSmall = ACT == SLORA_ACT_SILU ? 40.0f : 9.0f;
    static __device__ __forceinline__ float small(float x, float g)
    {
        if constexpr (ACT == SLORA_ACT_SILU) {
            const float t = g * -kAHigh, power = __builtin_amdgcn_exp2f(t);
            return x * (g * quotient(__builtin_fmaf(power, __builtin_fmaf(t, -0.693147180559945309417f, -g), power)));
        } else {
            return x * (g * quotient(Gate(g).z()));
        }
    }
    // All gates: z of -|g|, and for negative g 1 / (1 + 1 / z) = z / (1 + z), whose 2^n goes to x - there is a result wherever the product of all has one, though act(g) alone
    // may be below fp32's range.
    static __device__ __forceinline__ float any(float x, float g)
    {
        const Gate e(fminf(fabsf(g), 256.0f)); // (z is 0 from there on; NaN comes back with g)
        const bool negative = g < 0.0f;
        return __builtin_ldexpf(x, negative ? e.whole : 0) * (g * (quotient(e.z()) * (negative ? e.power : 1.0f)));
    }
};

// A piece whose gates are all small in all of the wavefront goes without the steps for the others (which round elsewhere: not by what is behind the row, so that a piece
// that is not whole takes them always).
template <int ACT, int DT>
__device__ __forceinline__ void gate_piece(float (&v)[kPiece], const u32x4 &gate, bool whole)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef Gate<DT, ACT> G;
    constexpr uint16_t kSmall = DT == SLORA_F16 ? __builtin_bit_cast(uint16_t, (_Float16)G::kSmall) : (uint16_t)(__builtin_bit_cast(uint32_t, G::kSmall) >> 16);
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, gate[i] & 0x7fff7fffu));
    float g[kPiece];
    widen8<DT>(gate, g);
    if (__builtin_amdgcn_ballot_w64(top[0] > kSmall || top[1] > kSmall || !whole) == 0) {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] = G::small(v[i], g[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] = G::any(v[i], g[i]);
    }
}

// Rows in 8 bits, or the gated product, as norms are taken: one row for the workgroup, or one for each of its wavefronts.
// Bound, plain rows: HBM (4096 of 5120 to 8 bits that are in no cache, 63 MB: 15.1 us = 4.2 TB/s; in the memory-side cache 12.1).  Gated ones: HBM beside the vector units - us to 8 bits with
// no gate / silu / gelu, 2048 rows of 20480 23.6 / 40.2 / 49.0, 3001 of 13008 23.1 / 39.5 / 47.1, of 13007 24.7 / 43.9 / 51.6 (the pieces of the last wavefront, above), and with u log2 e rounded as a
// number, which leaves fp32's accuracy, silu 40.7 / 38.6 / 40.9.  A kernel for each function: all three in one take more registers and 25.9 us without a gate, 41.2 with silu (3001 of 13008).
// With six wavefronts a SIMD asked for, rows of ten wavefronts run two to a compute unit: 2048 of 20480, silu 43.1 without, 40.2 with.
template <int DT, int ACT, int P, bool TAIL, bool ONCE>
__global__ __launch_bounds__(kRowThreads, P == 8 ? 4 : 6) void quantize_kernel(QuantizeArgs a, int waves)
{
    __shared__ uint32_t slots[1][kRowThreads / kWave];
    const int wave = wave_number();
    const int64_t t = row_number(waves, wave);
    if (t >= a.T) return;
    const Row<P, TAIL> r = row_of<P, TAIL>(a.width, waves);
    Team team{slots, waves, wave};
    u32x4 raw[P], gate[P];
    load16<ONCE>(r, a.x + t * a.x_stride, raw);
    if constexpr (ACT != SLORA_ACT_NONE) load16<ONCE>(r, a.gate + t * a.gate_stride, gate);
    float v[P][kPiece];
    const Row<P, TAIL> now = again(r);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        widen8<DT>(raw[p], v[p]);
        if constexpr (ACT != SLORA_ACT_NONE) gate_piece<ACT, DT>(v[p], gate[p], now.whole(p));
    }
    if (a.out.x) store16<DT>(r, a.out.x + t * a.out.x_stride, v);
    if (a.out.codes) store_codes(r, a.out, t, v, team);
}

// f(pieces of a lane, wavefronts of a row), by the width alone, so that a row's result does not depend on the others.
// Norms of rows of more than 2048 elements hold four pieces a lane, so that fewer wavefronts wait for each other.  us with two / four: 2048 rows of 4096 17.2 / 14.9, of
// 16384 64 / 51, 8192 of 8192 99 / 97, 777 of 5003 21.7 / 20.0, 8192 of 4096 without a norm behind the block 48 / 49; up to 1024 elements one
// wavefront has the row: 16384 of 1024 25 with two, 27 with four pieces, of 128 7.8 with one, 14 with four.
// Rows in 8 bits hold two up to 16384: 4096 of 5120 15 / 15, gated 3001 of 13007 44 / 47.
template <int MOST, typename F>
int32_t by_width(int width, F f)
{
    const int pieces = (width + kPiece - 1) / kPiece;
    auto waves = [&](int p) { return (pieces + p * kWave - 1) / (p * kWave); };
    if (waves(1) <= 1) return f(std::integral_constant<int, 1>{}, 1);
    if (waves(4) <= 1) return f(std::integral_constant<int, 2>{}, waves(2));
    if constexpr (MOST == 8) { // rows in 8 bits
        if (waves(2) <= 16) return f(std::integral_constant<int, 2>{}, waves(2));
        if (waves(4) > 16) return f(std::integral_constant<int, 8>{}, waves(8));
    }
    return f(std::integral_constant<int, 4>{}, waves(4));
}

// rows of one wavefront: four to a workgroup
struct Grid {
    dim3 blocks, threads;
    Grid(int32_t T, int waves) : threads(waves == 1 ? 4 * kWave : waves * kWave)
    {
        const int64_t n = waves == 1 ? ((int64_t)T + 3) / 4 : T;
        blocks = dim3((unsigned)std::min<int64_t>(n, kGridX), (unsigned)((n + kGridX - 1) / kGridX));
    }
};

template <typename F>
int32_t by_flag(bool flag, F f)
{
    return flag ? f(std::true_type{}) : f(std::false_type{});
}

} // namespace

int32_t launch_norm(const NormArgs &a, int32_t dtype, bool h32, void *stream)
{
    const int64_t bytes = (int64_t)a.T * a.width * ((h32 ? 4 : 2) + (a.block ? 2 : 0) + (a.gate && a.gate_stride ? 2 : 0)); // of rows
    return by_width<4>(a.width, [&](auto p, int waves) {
        return by_flag(a.width % kPiece != 0, [&](auto tail) {
            return by_flag(h32, [&](auto h) {
                return by_flag(bytes >= kOnceBytes, [&](auto once) {
                    const Grid g(a.T, waves);
                    if (dtype == SLORA_F16)
                        hipLaunchKernelGGL((norm_kernel<SLORA_F16, h.value, p.value, tail.value, once.value>), g.blocks, g.threads, 0, (hipStream_t)stream, a, waves);
                    else
                        hipLaunchKernelGGL((norm_kernel<SLORA_BF16, h.value, p.value, tail.value, once.value>), g.blocks, g.threads, 0, (hipStream_t)stream, a, waves);
                    return check_launch("norm");
                });
            });
        });
    });
}

int32_t launch_quantize(const QuantizeArgs &a, int32_t dtype, void *stream)
{
    const int64_t bytes = (int64_t)a.T * a.width * (a.gate ? 4 : 2);
    auto by_act = [&](auto f) {
        switch (a.act) {
        case SLORA_ACT_SILU: return f(std::integral_constant<int, SLORA_ACT_SILU>{});
        case SLORA_ACT_GELU: return f(std::integral_constant<int, SLORA_ACT_GELU>{});
        }
        return f(std::integral_constant<int, SLORA_ACT_NONE>{});
    };
    return by_width<8>(a.width, [&](auto p, int waves) {
        return by_flag(a.width % kPiece != 0, [&](auto tail) {
            return by_flag(bytes >= kOnceBytes, [&](auto once) {
                return by_act([&](auto act) {
                    const Grid g(a.T, waves);
                    if (dtype == SLORA_F16)
                        hipLaunchKernelGGL((quantize_kernel<SLORA_F16, act.value, p.value, tail.value, once.value>), g.blocks, g.threads, 0, (hipStream_t)stream, a, waves);
                    else
                        hipLaunchKernelGGL((quantize_kernel<SLORA_BF16, act.value, p.value, tail.value, once.value>), g.blocks, g.threads, 0, (hipStream_t)stream, a, waves);
                    return check_launch("quantize");
                });
            });
        });
    });
}

} // namespace slora
