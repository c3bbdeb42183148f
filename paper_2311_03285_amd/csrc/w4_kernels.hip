// gfx950 kernels of the products with 4-bit weights: packing, and y = x W for a few tokens.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "w4.hpp"

namespace slora {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------------------
// one workgroup per tile and chunk; thread = (lane, word)
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t *__restrict__ codes, const uint16_t *__restrict__ scales, const uint8_t *__restrict__ zeros,
                                                      uint8_t *__restrict__ packed, int outputs, int inputs, int group, int chunks, int unit, int64_t code_bytes,
                                                      int64_t units)
{
    const int64_t block = blockIdx.x;
    const int tile = (int)(block / chunks), chunk = (int)(block % chunks);
    const int lane = threadIdx.x / 4, word = threadIdx.x % 4;
    const int row = tile * kW4Rows + lane % 16, k0 = chunk * kW4Chunk + word * 32 + lane / 16 * 8;
    uint32_t u = 0;
    if (row < outputs && k0 < inputs) { // inputs is a multiple of 8
        const uint32_t v = *reinterpret_cast<const uint32_t *>(codes + (int64_t)row * (inputs / 2) + k0 / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) u |= ((v >> (4 * i)) & 15u) << (i < 4 ? 8 * i : 8 * (i - 4) + 4);
    }
    reinterpret_cast<uint32_t *>(packed)[block * 256 + threadIdx.x] = u;
    const int per = kW4Chunk / unit;
    if ((int)threadIdx.x < per * kW4Rows) {
        const int k = chunk * kW4Chunk + (int)threadIdx.x / kW4Rows * unit, r = tile * kW4Rows + threadIdx.x % kW4Rows;
        const bool in = r < outputs && k < inputs;
        const int64_t from = (int64_t)r * ((inputs + group - 1) / group) + k / group, at = block * per * kW4Rows + threadIdx.x;
        reinterpret_cast<uint16_t *>(packed + code_bytes)[at] = in ? scales[from] : (uint16_t)0;
        packed[code_bytes + 2 * units + at] = (in ? (zeros ? zeros[from] & 15 : 8) : 0) | 0x80; // the 8-bit float -z
    }
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
// Matrix instruction 16 x 16 x 32: tokens are rows, outputs columns; lane l = 16 g + n supplies inputs 8 g .. 8 g + 7 of row or column n,
// and receives rows 4 g .. 4 g + 3 of column n: a lane's sums are of ONE output, whose scale it needs.  Row m is token
// 4 (m % 4) + m / 4, so that up to four tokens are all in the first of the four rows that a lane receives.
// The bits of a code c = 0 .. 15, taken as an 8-bit float of four exponent and three mantissa bits (bias 7), are the
// number c * 2^-9 - the least exponent's numbers and the subnormal ones go up in even steps - so that one conversion of two bytes, with
// its scale of 512, makes two operands, exact in either 16-bit type.  (c - z) x is summed as c x and -z x, in one accumulator.
template <int DT>
struct Operand;
template <>
struct Operand<SLORA_F16> {
    typedef f16x8 type;
    static __device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f16x8 codes(uint32_t u)
    {
        const uint32_t lo = u & 0x0f0f0f0fu, hi = (u >> 4) & 0x0f0f0f0fu;
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true);
        return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ f16x8 all(uint32_t byte)
    {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(byte * 0x0101u, 512.0f, false);
        return __builtin_shufflevector(a, a, 0, 1, 0, 1, 0, 1, 0, 1);
    }
};
template <>
struct Operand<SLORA_BF16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ bf16x8 codes(uint32_t u)
    {
        const uint32_t lo = u & 0x0f0f0f0fu, hi = (u >> 4) & 0x0f0f0f0fu;
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true);
        return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ bf16x8 all(uint32_t byte)
    {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(byte * 0x0101u, 512.0f, false);
        return __builtin_shufflevector(a, a, 0, 1, 0, 1, 0, 1, 0, 1);
    }
};

__device__ __forceinline__ int token_of_row(int m) { return 4 * (m % 4) + m / 4; }

// Up to four tokens.  A workgroup = RT tiles of 16 outputs; its WV wavefronts take chunks of 128 inputs in turn, with the weights of the next ones and x of the
// next one under way, and are added in LDS.  Loads are not behind branches where others are waited for: the compiler would wait for all of them.
// Bound: HBM and the time to fill it: four of 4096 of 4096, one token 9.0 us = 3.8 TB/s, two of 20480 of 5120 28 us = 3.7 TB/s.
template <int DT, int RT, int WV, int U>
__global__ __launch_bounds__(WV *kWave) void w4_kernel(W4Args a, bool y16)
{
    typedef typename Operand<DT>::type operand;
    constexpr int kPer = kW4Chunk / U; // units of a chunk
    constexpr int kAhead = RT * kPer > 4 ? 2 : 4; // chunks of weights under way
    __shared__ float part[WV][4][RT * 16];
    int k = 0;
    while (k + 1 < a.n && (int)blockIdx.x >= a.m[k + 1].first) ++k;
    const W4Matrix &m = a.m[k];
    const int tiles = (m.outputs + kW4Rows - 1) / kW4Rows, chunks = m.chunks, inputs = m.inputs;
    const int tile0 = ((int)blockIdx.x - m.first) * RT;
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;

    float sum[RT] = {}; // of token g
    // (rows beyond the last token: the last once more, whose sums nobody takes)
    const uint16_t *const row = m.x + (int64_t)min(token_of_row(n), a.T - 1) * inputs;
    const uint8_t *const codes = m.codes, *const zeros = m.zeros;
    const uint16_t *const scales = m.scales;

    struct Chunk {
        u32x4 w[RT];
        uint16_t scale[RT][kPer];
        uint8_t zero[RT][kPer];
    } ring[kAhead];
    u32x4 x[2][4];
    auto fetch_w = [&](Chunk &next, int c) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int64_t tile = (int64_t)min(tile0 + r, tiles - 1) * chunks + c;
            next.w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + tile * 1024 + (uint32_t)lane * 16));
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                next.scale[r][u] = scales[(tile * kPer + u) * kW4Rows + (uint32_t)n];
                next.zero[r][u] = zeros[(tile * kPer + u) * kW4Rows + (uint32_t)n];
            }
        }
    };
    auto fetch_x = [&](u32x4 (&xn)[4], int c) {
#pragma unroll
        for (int s = 0; s < 4; ++s) xn[s] = *reinterpret_cast<const u32x4 *>(row + min(c * kW4Chunk + s * 32 + g * 8, inputs - 8));
    };
    auto work = [&](const Chunk &now, u32x4 (&xs)[4], int c) {
        if ((c + 1) * kW4Chunk > inputs) { // inputs that there are not
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (c * kW4Chunk + s * 32 + g * 8 >= inputs) xs[s] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                f32x4 acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                const operand z = Operand<DT>::all(now.zero[r][u]);
#pragma unroll
                for (int s = u * (U / 32); s < (u + 1) * (U / 32); ++s) {
                    const operand xo = __builtin_bit_cast(operand, xs[s]);
                    acc = Operand<DT>::mfma(xo, Operand<DT>::codes(now.w[r][s]), acc);
                    acc = Operand<DT>::mfma(xo, z, acc);
                }
                sum[r] = __builtin_fmaf(acc[0], widen<DT>(now.scale[r][u]), sum[r]);
            }
    };
    if (wave < chunks) {
        const int mine = (chunks - wave + WV - 1) / WV; // chunks of this wavefront
        auto chunk = [&](int i) { return wave + min(i, mine - 1) * WV; };
        fetch_x(x[0], chunk(0));
        int i = 0;
        if (mine > kAhead) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) fetch_w(ring[k], chunk(k));
            for (; i + kAhead < mine; i += kAhead) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    fetch_x(x[(k + 1) % 2], chunk(i + k + 1));
                    work(ring[k], x[k % 2], chunk(i + k));
                    fetch_w(ring[k], chunk(i + k + kAhead));
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k < mine) fetch_w(ring[k], chunk(k));
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= mine) break;
            fetch_x(x[(k + 1) % 2], chunk(i + k + 1));
            work(ring[k], x[k % 2], chunk(i + k));
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) part[wave][g][r * 16 + n] = sum[r];
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 16 * a.T; i += WV * kWave) {
        const int r = i % (RT * 16), t = i / (RT * 16), o = tile0 * kW4Rows + r;
        if (o >= m.outputs) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WV; ++w) v += part[w][t][r];
        const int64_t at = (int64_t)t * m.outputs + o;
        if (y16)
            static_cast<uint16_t *>(m.y)[at] = narrow<DT>(v);
        else
            static_cast<float *>(m.y)[at] = v;
    }
}

// More tokens: x, which every tile of outputs needs, is shared.  Eight wavefronts in TEAMS teams, which take chunks in turn; those of a team have
// RT tiles of outputs each and read their chunk of x from LDS, where they have put it together (a row is 256
// bytes, its pieces of 16 bytes permuted by its number, so that the 16 rows of an operand are in different banks).  While a chunk is
// worked on, the team's next one goes from registers to the other buffer, the one after that from memory to
// registers; the barrier between chunks waits for LDS alone.
// Two of 20480 of 5120, 32 tokens 37 - 39 us = 340 - 360 TFLOP/s and 3.0 - 3.2 TB/s; three of 5003 of 3080, 67 tokens, groups of 32 25 - 26 us.  Bound: no unit alone - of the former's
// cycles the vector units are busy for 35 % (at four an instruction), the matrix units, half of whose work takes the zeros off, for 26 %.
constexpr int kWideThreads = 8 * kWave;

__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int DT, int TEAMS, int RT, int NT, int U>
__global__ __launch_bounds__(kWideThreads, TEAMS == 2 && RT == 1 && NT <= 2 && (U > 32 || NT == 1) ? 6 : 2) void w4_wide_kernel(W4Args a, bool y16)
{
    typedef typename Operand<DT>::type operand;
    constexpr int kPer = kW4Chunk / U, kRows = NT * 16, kPieces = kW4Chunk / 8;
    // Chunks of weights under way.  Two, and with them registers for three workgroups of a compute unit, are as fast as four and two workgroups, or faster: two of
    // 20480 of 5120, 32 tokens 39.2 us with two, 44.4 with four, where two at a time go through 640 workgroups in one round and a quarter.
    constexpr int kAhead = 2;
    constexpr int kMembers = 8 / TEAMS;     // wavefronts of a team,
    constexpr int kPuts = NT * 4 / kMembers; // each of which puts four rows at a time into LDS, so often
    constexpr int kStage = kRows * kPieces, kMerge = 8 * RT * NT * kWave; // pieces of 16 bytes
    __shared__ u32x4 lds[TEAMS * 2 * kStage > kMerge ? TEAMS * 2 * kStage : kMerge];
    int k = 0;
    while (k + 1 < a.n && (int)blockIdx.x >= a.m[k + 1].first) ++k;
    const W4Matrix &m = a.m[k];
    const int tiles = (m.outputs + kW4Rows - 1) / kW4Rows, chunks = m.chunks, inputs = m.inputs;
    const int wave = wave_number(), team = wave / kMembers, rw = wave % kMembers, lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    const int tile0 = (((int)blockIdx.x - m.first) * kMembers + rw) * RT, t0 = blockIdx.y * kRows;
    u32x4 *const stage = lds + team * 2 * kStage;
    const uint8_t *const codes = m.codes, *const zeros = m.zeros;
    const uint16_t *const scales = m.scales;

    f32x4 sum[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // this thread's pieces of a chunk of x: number n of rows 4 (kMembers j + rw) + g (rows beyond the last token: the last once more, whose sums nobody takes)
    auto row_of = [&](int j) { return 4 * (kMembers * j + rw) + g; };
    const uint16_t *row[kPuts];
#pragma unroll
    for (int j = 0; j < kPuts; ++j) row[j] = m.x + (int64_t)min(t0 + row_of(j) / 16 * 16 + token_of_row(row_of(j) % 16), a.T - 1) * inputs;
    u32x4 xr[kPuts];
    auto fetch_x = [&](int c) {
        const int at = min(c * kW4Chunk + n * 8, inputs - 8);
#pragma unroll
        for (int j = 0; j < kPuts; ++j) xr[j] = *reinterpret_cast<const u32x4 *>(row[j] + at);
    };
    auto put_x = [&](int buffer, int c) {
        if ((c + 1) * kW4Chunk > inputs) { // inputs that there are not
            const bool in = c * kW4Chunk + n * 8 < inputs;
#pragma unroll
            for (int j = 0; j < kPuts; ++j) xr[j] = in ? xr[j] : u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int j = 0; j < kPuts; ++j) stage[buffer * kStage + row_of(j) * kPieces + (n ^ (row_of(j) % 16))] = xr[j];
    };
    const u32x4 *take[4]; // this lane's piece of step s
#pragma unroll
    for (int s = 0; s < 4; ++s) take[s] = stage + n * kPieces + ((4 * s + g) ^ n);
    struct Chunk {
        u32x4 w[RT];
        uint16_t scale[RT][kPer];
        uint8_t zero[RT][kPer];
    } ring[kAhead];
    auto fetch_w = [&](Chunk &next, int c) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int64_t tile = (int64_t)min(tile0 + r, tiles - 1) * chunks + c;
            next.w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + tile * 1024 + (uint32_t)lane * 16));
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                next.scale[r][u] = scales[(tile * kPer + u) * kW4Rows + (uint32_t)n];
                next.zero[r][u] = zeros[(tile * kPer + u) * kW4Rows + (uint32_t)n];
            }
        }
    };
    // both teams go through the same number of barriers
    const int turns = (chunks + TEAMS - 1) / TEAMS;
    auto chunk_of = [&](int turn) { return min(turn * TEAMS + team, chunks - 1); };
    // (loads in the order of the loop below, which waits for them by their number)
    fetch_x(chunk_of(0));
#pragma unroll
    for (int k = 0; k + 1 < kAhead; ++k) fetch_w(ring[k], chunk_of(k));
    put_x(0, chunk_of(0));
    fetch_x(chunk_of(1));
    fetch_w(ring[kAhead - 1], chunk_of(kAhead - 1));
    lds_barrier();
    for (int turn0 = 0; turn0 < turns; turn0 += kAhead) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) { // (kAhead is even: turn k of them reads buffer k % 2)
            const int turn = turn0 + k;
            if (turn >= turns) break;
            put_x((k + 1) % 2, chunk_of(turn + 1));
            fetch_x(chunk_of(turn + 2));
            Chunk &now = ring[k];
            if (turn * TEAMS + team < chunks) {
#pragma unroll
                for (int u = 0; u < kPer; ++u) {
                    operand xo[U / 32][NT];
#pragma unroll
                    for (int s = 0; s < U / 32; ++s)
#pragma unroll
                        for (int t = 0; t < NT; ++t) xo[s][t] = __builtin_bit_cast(operand, take[u * (U / 32) + s][k % 2 * kStage + t * 16 * kPieces]);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        f32x4 acc[NT];
                        const operand z = Operand<DT>::all(now.zero[r][u]);
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int s = 0; s < U / 32; ++s) {
                            const operand cw = Operand<DT>::codes(now.w[r][u * (U / 32) + s]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[t] = Operand<DT>::mfma(xo[s][t], cw, acc[t]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[t] = Operand<DT>::mfma(xo[s][t], z, acc[t]);
                        }
                        const float scale = widen<DT>(now.scale[r][u]);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[r][t][i] = __builtin_fmaf(acc[t][i], scale, sum[r][t][i]);
                    }
                }
            }
            fetch_w(now, chunk_of(turn + kAhead));
            lds_barrier();
        }
    }
    // the other teams' sums to the first
    f32x4 *merge = reinterpret_cast<f32x4 *>(lds);
    if (team > 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) merge[(wave * RT * NT + r * NT + t) * kWave + lane] = sum[r][t];
    }
    lds_barrier();
    if (team > 0) return;
#pragma unroll
    for (int k = 1; k < TEAMS; ++k)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[r][t] += merge[((wave + k * kMembers) * RT * NT + r * NT + t) * kWave + lane];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x4 v = sum[r][t];
            const int o = (tile0 + r) * kW4Rows + n;
            if (o >= m.outputs) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int token = t0 + t * 16 + 4 * i + g;
                if (token >= a.T) continue;
                const int64_t at = (int64_t)token * m.outputs + o;
                if (y16)
                    static_cast<uint16_t *>(m.y)[at] = narrow<DT>(v[i]);
                else
                    static_cast<float *>(m.y)[at] = v[i];
            }
        }
}

// workgroups of `each` tiles of outputs
int64_t share_out(W4Args &a, int each)
{
    int64_t groups = 0;
    for (int32_t k = 0; k < a.n; ++k) {
        a.m[k].first = (int32_t)groups;
        groups += ((int64_t)a.m[k].outputs + kW4Rows * each - 1) / (kW4Rows * each);
    }
    return groups;
}

template <int DT, int RT, int WV, int U>
int32_t launch(W4Args &a, bool y16, void *stream)
{
    const int64_t groups = share_out(a, RT);
    hipLaunchKernelGGL((w4_kernel<DT, RT, WV, U>), dim3((unsigned)groups), dim3(WV * kWave), 0, (hipStream_t)stream, a, y16);
    return check_launch("w4");
}

template <int DT, int TEAMS, int RT, int NT, int U>
int32_t launch_wide(W4Args &a, bool y16, void *stream)
{
    const int64_t groups = share_out(a, 8 / TEAMS * RT), blocks = ((int64_t)a.T + NT * 16 - 1) / (NT * 16);
    if (blocks > 65535) return fail(SLORA_ERANGE, "T=%d tokens are too many for one call", a.T);
    hipLaunchKernelGGL((w4_wide_kernel<DT, TEAMS, RT, NT, U>), dim3((unsigned)groups, (unsigned)blocks), dim3(kWideThreads), 0, (hipStream_t)stream, a, y16);
    return check_launch("w4_wide");
}

// Teams: the fewer workgroups of 16 outputs there are, the more of its eight wavefronts share out a workgroup's inputs.  us with 2, 4, 8 teams: 1024
// outputs of 8192 inputs, two matrices, 32 tokens 23.2 / 15.2 / 13.0; 4096 of 4096, 32 tokens 12.7 / 10.3 / 10.0; 8192 of 8192, 32 tokens
// 22.7 / 16.3 / 24.5; four of 4096 of 4096, 16 tokens 12.0 / 12.5 / 17.8.  (Eight teams' x of more than 32 tokens does not fit LDS.)
// Two tiles of outputs a wavefront where x is read for 33 - 48 tokens, from 1536 workgroups of one on.  us with one / two: six of 4096 of 4096, 40 tokens 26.1 / 24.6; three
// of 8192 of 8192, 48 tokens 51.5 / 47.6; three of 4096 of 4096, 96 tokens 26.2 / 24.1; 13000 of 2048, 80 tokens, groups of 32 18.6 / 18.2; four of
// 16384 of 4096, 130 tokens 164 / 156; two of 20480 of 5120, 70 tokens 85.7 / 86.3.  Below: 20480 of 5120, 40 tokens (1280) 29.7 / 27.8, but 8192 of 8192, 90 tokens, groups of
// 32 (1024) 34.3 / 52.4.  Where x is read for 64 tokens, four of 8192 of 8192 69.6 / 71.8, and for 32, two of 20480 of 5120 42.0 / 48.0.
template <int DT, int U, int NT>
int32_t wide(W4Args &a, int64_t tiles, bool y16, void *stream)
{
    const int64_t groups = tiles * (((int64_t)a.T + NT * 16 - 1) / (NT * 16)); // of 16 outputs and NT * 16 tokens
    if constexpr (NT <= 2) {
        if (groups <= 256) return launch_wide<DT, 8, 1, NT, U>(a, y16, stream);
    }
    if (groups <= 512) return launch_wide<DT, 4, 1, NT, U>(a, y16, stream);
    if constexpr (NT == 3) {
        if (groups >= 1536) return launch_wide<DT, 2, 2, NT, U>(a, y16, stream);
    }
    return launch_wide<DT, 2, 1, NT, U>(a, y16, stream);
}

// Up to four tokens read x for themselves.  us, w4_kernel / w4_wide_kernel: 4096 of 4096, one token 4.8 / 6.0, 8192 of 8192 9.8 / 12.0, four of 4096 of
// 4096 9.8 / 11.9, two of 20480 of 5120 28.0 / 27.0; of 8 tokens the second one is as fast or faster (8192 of 8192 14.4 / 12.9).
template <int DT, int U>
int32_t by_tokens(W4Args &a, bool y16, void *stream)
{
    int64_t tiles = 0;
    for (int32_t k = 0; k < a.n; ++k) tiles += (a.m[k].outputs + kW4Rows - 1) / kW4Rows;
    if (a.T <= 4) {
        // two tiles share x; us with one / two: 4096 of 4096 4.7 / 5.5, 8192 of 8192 10.4 / 9.3; eight / four wavefronts: two of 20480 of 5120 33.5 / 28.0,
        // four of 4096 of 4096 9.4 / 10.1
        if (tiles >= 2048) return launch<DT, 2, 4, U>(a, y16, stream);
        if (tiles >= 512) return launch<DT, 2, 8, U>(a, y16, stream);
        return launch<DT, 1, 8, U>(a, y16, stream);
    }
    const int32_t rows = (a.T - 1) / 16 + 1, blocks = (rows + 3) / 4;
    switch ((rows + blocks - 1) / blocks) {
    case 1: return wide<DT, U, 1>(a, tiles, y16, stream);
    case 2: return wide<DT, U, 2>(a, tiles, y16, stream);
    case 3: return wide<DT, U, 3>(a, tiles, y16, stream);
    }
    return wide<DT, U, 4>(a, tiles, y16, stream);
}

} // namespace

int32_t launch_w4_pack(const slora_w4 *w, const void *codes, const void *scales, const uint8_t *zeros, void *packed, void *stream)
{
    const int64_t blocks = (int64_t)w->tiles * w->chunks;
    if (blocks > INT32_MAX) return fail(SLORA_ERANGE, "a matrix of %d x %d is too large", w->outputs, w->inputs);
    hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, static_cast<const uint8_t *>(codes),
                       static_cast<const uint16_t *>(scales), zeros, static_cast<uint8_t *>(packed), w->outputs, w->inputs, w->group, w->chunks, w->unit,
                       w->code_bytes(), w->units());
    return check_launch("w4_pack");
}

int32_t launch_w4(const slora_w4 *const *w, W4Args &a, bool y16, void *stream)
{
    auto by_unit = [&](auto dt) -> int32_t {
        switch (w[0]->unit) {
        case 128: return by_tokens<dt.value, 128>(a, y16, stream);
        case 64: return by_tokens<dt.value, 64>(a, y16, stream);
        }
        return by_tokens<dt.value, 32>(a, y16, stream);
    };
    return w[0]->dtype == SLORA_F16 ? by_unit(std::integral_constant<int, SLORA_F16>{}) : by_unit(std::integral_constant<int, SLORA_BF16>{});
}

} // namespace slora
