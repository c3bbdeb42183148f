// gfx950 kernels of the products with 8-bit weights: packing, and y = x W for few tokens and for many.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "w8.hpp"

namespace slora {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------------------
// a wavefront per block of 16 outputs x 64 inputs
__global__ __launch_bounds__(256) void w8_pack_kernel(const int8_t *__restrict__ codes, const float *__restrict__ scales, int8_t *__restrict__ packed, int outputs, int inputs,
                                                      int chunks, int64_t blocks)
{
    const int64_t block = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (block >= blocks) return;
    const int64_t tile = block / chunks;
    const int chunk = (int)(block % chunks), lane = threadIdx.x % kWave;
    const int64_t row = tile * kW8Rows + lane % 16;
    const int k0 = chunk * kW8Chunk + lane / 16 * 16;
    uint32_t u[4] = {};
    if (row < outputs) {
        const int8_t *from = codes + row * inputs + k0;
        if (k0 + 16 <= inputs && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
            const i32x4 v = *reinterpret_cast<const i32x4 *>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = (uint32_t)v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k0 + i < inputs) u[i / 4] |= (uint32_t)(uint8_t)from[i] << (8 * (i % 4));
        }
    }
    reinterpret_cast<i32x4 *>(packed)[block * kWave + lane] = i32x4{(int)u[0], (int)u[1], (int)u[2], (int)u[3]};
    if (chunk == 0 && lane < kW8Rows) reinterpret_cast<float *>(packed + blocks * kW8Block)[row] = row < outputs ? scales[row] : 0.0f;
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
// Matrix instructions 16 x 16 x 64 and 32 x 32 x 32 on 8-bit integers.  A lane supplies 16 bytes of one row or
// column; which inputs they are does not matter as long as it is the same ones for x and for the weights.
__device__ __forceinline__ i32x4 mfma16(const i32x4 &a, const i32x4 &b, const i32x4 &c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
__device__ __forceinline__ i32x16 mfma32(const i32x4 &a, const i32x4 &b, const i32x16 &c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }

__device__ __forceinline__ i32x4 load16b(const int8_t *p) { return *reinterpret_cast<const i32x4 *>(p); }

// Y: 0 fp32, else 1 + the 16-bit type.  The sum, exact so far, is rounded to fp32 and multiplied by both scales there; the product of the scales
// alone could leave the range that the three have.
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale) { return (float)sum * x_scale * w_scale; }
template <int Y>
__device__ __forceinline__ void store_y(void *y, int64_t at, float v)
{
    if constexpr (Y == 0)
        static_cast<float *>(y)[at] = v;
    else
        static_cast<uint16_t *>(y)[at] = narrow<Y - 1>(v);
}

__device__ __forceinline__ int matrix_of(const W8Args &a, int block)
{
    int k = 0;
    while (k + 1 < a.n && block >= a.m[k + 1].first) ++k;
    return k;
}

__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Few tokens: weights go from memory to the matrix instruction's registers.  A workgroup = RT tiles of 16 outputs and NT * 16 tokens; its
// wavefronts take chunks of inputs in turn and are added up in LDS.
constexpr int kFewWaves = 8;
template <int RT, int NT, int Y>
__global__ __launch_bounds__(kFewWaves *kWave) void w8_few_kernel(W8Args a)
{
    constexpr int kAhead = 4; // chunks of weights under way
    __shared__ int part[kFewWaves][RT * NT][4][kWave];
    const W8Matrix &m = a.m[matrix_of(a, blockIdx.x)];
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    const int tile0 = ((int)blockIdx.x - m.first) * RT, t0 = blockIdx.y * NT * 16, chunks = m.chunks, x_last = m.x_last;

    i32x4 sum[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[r][t] = i32x4{0, 0, 0, 0};
    const int8_t *row[NT], *codes[RT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row[t] = m.x + (int64_t)min(t0 + t * 16 + n, a.T - 1) * m.x_stride;
#pragma unroll
    for (int r = 0; r < RT; ++r) codes[r] = m.codes + (int64_t)min(tile0 + r, m.tiles - 1) * chunks * kW8Block + lane * 16;

    struct Chunk {
        i32x4 w[RT], x[NT];
    } ring[kAhead];
    // (inputs behind the last: weights of 0)
    auto fetch = [&](Chunk &to, int c) {
#pragma unroll
        for (int r = 0; r < RT; ++r) to.w[r] = __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(codes[r] + (int64_t)c * kW8Block));
#pragma unroll
        for (int t = 0; t < NT; ++t) to.x[t] = load16b(row[t] + min(c * kW8Chunk + g * 16, x_last));
    };
    auto work = [&](const Chunk &now) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[r][t] = mfma16(now.x[t], now.w[r], sum[r][t]);
    };
    if (wave < chunks) {
        const int mine = (chunks - wave + kFewWaves - 1) / kFewWaves; // chunks of this wavefront
        auto chunk = [&](int i) { return wave + min(i, mine - 1) * kFewWaves; };
#pragma unroll
        for (int k = 0; k < kAhead; ++k) fetch(ring[k], chunk(k));
        int i = 0;
        for (; i + kAhead < mine; i += kAhead) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                work(ring[k]);
                fetch(ring[k], chunk(i + k + kAhead));
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k < mine) work(ring[k]);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][r * NT + t][i][lane] = sum[r][t][i];
    __syncthreads();
    const int tokens = min(NT * 16, a.T - t0);
    for (int w = threadIdx.x; w < RT * 16 * tokens; w += kFewWaves * kWave) {
        const int r = w % (RT * 16), t = w / (RT * 16), o = tile0 * kW8Rows + r;
        if (o >= m.outputs) continue;
        int total = 0;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) total += part[k][r / 16 * NT + t / 16][t % 4][t % 16 / 4 * 16 + r % 16];
        store_y<Y>(m.y, (int64_t)(t0 + t) * m.y_stride + o, scaled(total, m.x_scales[t0 + t], m.scales[o]));
    }
}

// Many tokens: a workgroup of four wavefronts, two by two, takes 2 * MO * 32 outputs and 2 * MT * 32 tokens, in stages of 128 inputs that go through LDS: two
// buffers, one that is read while the next stage is written to the other, whose bytes have come from memory a stage before.
// LDS holds units of 16 bytes, [16 rows][chunk of 64][piece of 16][row]: an operand's read is 16 lanes of neighbouring units.  Weights lie so in memory.
// Rows of x come in eights of pieces (128 bytes); a row's place among 16 is permuted by the piece's number, so that the lanes that write
// eights or sixteens of pieces are in different banks.
// Outputs are the rows of the matrix instruction here, so that a lane has four neighbouring ones of a token, which go to LDS together and from there
// to y in rows.
constexpr int kTileThreads = 256, kStageBytes = 2 * kW8Chunk;
constexpr int kRaw = 0x00027000; // a buffer of 32-bit words, without a format

template <int MO, int MT>
constexpr int tile_lds(int y_bytes) // stages, or the outputs of 32 tokens of each wavefront
{
    return std::max(2 * (2 * MO * 32 + 2 * MT * 32) * kStageBytes, 4 * 32 * (MO * 32 * y_bytes + 16));
}

template <int MO, int MT, int Y>
__global__ __launch_bounds__(kTileThreads, MO * MT > 4 ? 1 : 2) void w8_tile_kernel(W8Args a)
{
    constexpr int BO = 2 * MO * 32, BT = 2 * MT * 32, kUnits = 8; // units of a row and stage
    constexpr int kPutsX = BT * kUnits / kTileThreads, kPutsW = BO * kUnits / kTileThreads, kPuts = kPutsX + kPutsW, kQuarter = kPuts / 4;
    constexpr int kReads = MT + MO, kBeside = kReads + 2 * kQuarter; // of a step
    extern __shared__ i32x4 lds[]; // [2][BT * kUnits], [2][BO * kUnits]
    i32x4 *const lds_x = lds, *const lds_w = lds + 2 * BT * kUnits;
    const int k = matrix_of(a, blockIdx.x);
    const W8Matrix &m = a.m[k];
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 32, h = lane / 32;
    const int wt = wave / 2, wo = wave % 2;

    const int tiles_o = (m.outputs + BO - 1) / BO, block = (int)blockIdx.x - m.first;
    const int t0 = block / tiles_o * BT, o0 = block % tiles_o * BO;

    // This thread's units of a stage: of x, number threadIdx % 8 of rows 32 j + threadIdx / 8; of tiles of 16 outputs 2 j + threadIdx / 128.  Where a row or the last
    // tile ends inside a stage, loads go on into what is behind, whose weights are 0, as far as the rows of the workgroup, or the codes, reach; loads beyond are 0.
    const int stages = m.chunks / 2, rows = min(BT, a.T - t0), tiles = min(BO / kW8Rows, m.tiles - o0 / kW8Rows);
    const auto x_rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(m.x + (int64_t)t0 * m.x_stride), 0, (rows - 1) * m.x_stride + m.x_last + 16, kRaw);
    const auto w_tiles = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(m.codes + (int64_t)(o0 / kW8Rows) * m.chunks * kW8Block), 0, tiles * m.chunks * kW8Block, kRaw);
    const int piece = threadIdx.x % 8, row0 = threadIdx.x / 8;
    auto place = [](int p) { return 2 * p ^ p / 4; }; // permutes the rows of a piece
    const int x_put = (row0 / 16 * 2 + piece / 4) * 64 + piece % 4 * 16 + ((row0 % 16) ^ place(piece)); // row0 + 32 j: 256 j units on
    int at[kPuts];
#pragma unroll
    for (int j = 0; j < kPutsX; ++j) at[j] = min(row0 + 32 * j, rows - 1) * m.x_stride + piece * 16;
#pragma unroll
    for (int j = 0; j < kPutsW; ++j) at[kPutsX + j] = min(2 * j + (int)threadIdx.x / 128, tiles - 1) * m.chunks * kW8Block + (int)threadIdx.x % 128 * 16;
    i32x4 raw[kPuts];
    auto fetch = [&](int j, int s) {
        raw[j] = j < kPutsX ? __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(x_rows, at[j], s * kStageBytes, 0))
                            : __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_tiles, at[j], s * 2 * kW8Block, 0));
    };
    auto put = [&](int j, int buffer) {
        if (j < kPutsX)
            lds_x[buffer * BT * kUnits + x_put + j * 256] = raw[j];
        else
            lds_w[buffer * BO * kUnits + threadIdx.x + (j - kPutsX) * 256] = raw[j];
    };
    // units of step ks (32 inputs) of row n: piece 2 ks + h
    const i32x4 *take_x[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) take_x[ks] = lds_x + (wt * MT * 2 + n / 16) * 128 + ks / 2 * 64 + (2 * ks + h) % 4 * 16 + ((n % 16) ^ place(2 * ks + h));
    const i32x4 *const take_w = lds_w + (wo * MO * 2 + n / 16) * 128 + h * 16 + n % 16;
    i32x4 xf[2][MT], wf[2][MO];
    auto read = [&](int i, int buffer, int ks) {
        if (i < MT)
            xf[ks % 2][i] = take_x[ks][buffer * BT * kUnits + i * 256];
        else
            wf[ks % 2][i - MT] = take_w[buffer * BO * kUnits + (i - MT) * 256 + ks * 32];
    };
    i32x16 sum[MO][MT];
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[i][j][e] = 0;

    // A quarter of a stage's units is written in each step.  The buffer that step 3 of a stage leaves takes the first quarter of the stage after next there, and the other
    // ones in the steps after; registers that have been written take the stage after.
#pragma unroll
    for (int j = 0; j < kPuts; ++j) fetch(j, 0);
#pragma unroll
    for (int j = 0; j < kPuts; ++j) {
        put(j, 0);
        fetch(j, min(1, stages - 1));
    }
#pragma unroll
    for (int j = 0; j < kQuarter; ++j) {
        put(j, 1);
        fetch(j, min(2, stages - 1));
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(i, 0, 0);
    for (int s = 0; s < stages; ++s) {
        const int buffer = s % 2;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (ks == 3) lds_barrier(); // the next stage is in the other buffer; nobody reads this one any more
            // (behind the last stage: the last once more, which nobody multiplies)
            const int to = ks < 3 ? buffer ^ 1 : buffer, quarter = (ks + 1) % 4, next = min(s + (ks < 3 ? 2 : 3), stages - 1);
#pragma unroll
            for (int p = 0; p < MO * MT; ++p) {
                sum[p / MT][p % MT] = mfma32(wf[ks % 2][p / MT], xf[ks % 2][p % MT], sum[p / MT][p % MT]);
                // beside each product: operands of the next step first, then units to LDS and from memory in turn
#pragma unroll
                for (int o = p * kBeside / (MO * MT); o < (p + 1) * kBeside / (MO * MT); ++o) {
                    const int j = quarter * kQuarter + (o - kReads) / 2;
                    if (o < kReads)
                        read(o, ks < 3 ? buffer : buffer ^ 1, (ks + 1) % 4);
                    else if ((o - kReads) % 2 == 0)
                        put(j, to);
                    else
                        fetch(j, next);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    lds_barrier();
    // Rows 8 b + 4 h + i of column n are register 4 b + i.  A wavefront's outputs of 32 tokens go through LDS, a token's 16 bytes apart from the next one's end.
    typedef typename std::conditional<Y == 0, float, uint16_t>::type Out;
    constexpr int kRow = MO * 32 * (int)sizeof(Out), kPitch = kRow + 16, kLanes = kRow / 16, kEach = 16 / (int)sizeof(Out);
    char *const stage = reinterpret_cast<char *>(lds) + wave * 32 * kPitch;
    const int ow = o0 + wo * MO * 32;
    const bool aligned = m.y_stride % kEach == 0;
    Out *const y = static_cast<Out *>(m.y);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int tw = t0 + (wt * MT + j) * 32;
        const float x_scale = m.x_scales[min(tw + n, a.T - 1)];
#pragma unroll
        for (int i = 0; i < MO; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 w_scale = *reinterpret_cast<const f32x4 *>(m.scales + min(ow + i * 32 + 8 * b + 4 * h, m.tiles * kW8Rows - 4));
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = scaled(sum[i][j][4 * b + e], x_scale, w_scale[e]);
                char *const to = stage + n * kPitch + (i * 32 + 8 * b + 4 * h) * sizeof(Out);
                if constexpr (Y == 0)
                    *reinterpret_cast<f32x4 *>(to) = f32x4{v[0], v[1], v[2], v[3]};
                else
                    *reinterpret_cast<u32x2 *>(to) = u32x2{(uint32_t)narrow<Y - 1>(v[0]) | (uint32_t)narrow<Y - 1>(v[1]) << 16,
                                                           (uint32_t)narrow<Y - 1>(v[2]) | (uint32_t)narrow<Y - 1>(v[3]) << 16};
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
        if (aligned) {
#pragma unroll
            for (int r = 0; r < 32; r += kWave / kLanes) {
                const int row = r + lane / kLanes, o = ow + lane % kLanes * kEach;
                const i32x4 v = *reinterpret_cast<const i32x4 *>(stage + row * kPitch + lane % kLanes * 16);
                if (tw + row >= a.T) continue;
                Out *const to = y + (int64_t)(tw + row) * m.y_stride + o;
                if (o + kEach <= m.outputs) {
                    *reinterpret_cast<i32x4 *>(to) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < kEach; ++e)
                        if (o + e < m.outputs) to[e] = __builtin_bit_cast(Out, (typename std::conditional<Y == 0, int, uint16_t>::type)((uint32_t)v[e * (int)sizeof(Out) / 4] >> (Y == 0 ? 0 : e % 2 * 16)));
                }
            }
        } else {
            for (int r = 0; r < 32; ++r) {
                if (tw + r >= a.T) break;
#pragma unroll
                for (int e = 0; e < MO * 32; e += kWave) {
                    const int o = ow + e + lane;
                    if (o < m.outputs) y[(int64_t)(tw + r) * m.y_stride + o] = *reinterpret_cast<const Out *>(stage + r * kPitch + (e + lane) * sizeof(Out));
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    }
}

constexpr int64_t kMostThreads = (int64_t(1) << 32) - 1; // of a grid

// workgroups of `each` outputs, `blocks` of tokens; returns how many, which may be too many for a grid
int64_t share_out(W8Args &a, int each, int64_t blocks)
{
    int64_t groups = 0;
    for (int32_t k = 0; k < a.n; ++k) {
        a.m[k].first = (int32_t)std::min<int64_t>(groups, INT32_MAX);
        groups += ((int64_t)a.m[k].outputs + each - 1) / each * blocks;
    }
    return groups;
}

template <int RT, int NT, int Y>
int32_t launch_few(W8Args &a, void *stream)
{
    const int64_t groups = share_out(a, RT * kW8Rows, 1), blocks = ((int64_t)a.T + NT * 16 - 1) / (NT * 16);
    if (groups * kFewWaves * kWave > kMostThreads || blocks > 65535) return fail(SLORA_ERANGE, "T=%d tokens are too many for one call", a.T);
    hipLaunchKernelGGL((w8_few_kernel<RT, NT, Y>), dim3((unsigned)groups, (unsigned)blocks), dim3(kFewWaves * kWave), 0, (hipStream_t)stream, a);
    return check_launch("w8_few");
}

template <int MO, int MT, int Y>
int32_t launch_tile(W8Args &a, void *stream)
{
    constexpr int BO = 2 * MO * 32, BT = 2 * MT * 32, kLds = tile_lds<MO, MT>(Y == 0 ? 4 : 2);
    const int64_t groups = share_out(a, BO, ((int64_t)a.T + BT - 1) / BT);
    if (groups * kTileThreads > kMostThreads) return fail(SLORA_ERANGE, "T=%d tokens are too many for one call", a.T);
    if (kLds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&w8_tile_kernel<MO, MT, Y>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return fail(SLORA_EHIP, "hipFuncSetAttribute(LDS size): %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL((w8_tile_kernel<MO, MT, Y>), dim3((unsigned)groups), dim3(kTileThreads), kLds, (hipStream_t)stream, a);
    return check_launch("w8_tile");
}

template <int Y>
int32_t by_tokens(W8Args &a, void *stream)
{
    if (a.T <= 16) return launch_few<1, 1, Y>(a, stream);
    if (a.T <= 32) return launch_few<1, 2, Y>(a, stream);
    if (a.T <= 64) return launch_few<1, 4, Y>(a, stream);
    int64_t tiles = 0; // of 256 x 256
    for (int32_t k = 0; k < a.n; ++k) tiles += ((int64_t)a.m[k].outputs + 255) / 256 * (((int64_t)a.T + 255) / 256);
    if (tiles >= 200) return launch_tile<4, 4, Y>(a, stream);
    return launch_tile<2, 2, Y>(a, stream);
}

} // namespace

int32_t launch_w8_pack(const slora_w8 *w, const int8_t *codes, const float *scales, void *packed, void *stream)
{
    const int64_t blocks = (int64_t)w->tiles * w->chunks, groups = (blocks + 3) / 4;
    if (groups * 256 > kMostThreads) return fail(SLORA_ERANGE, "a matrix of %d x %d is too large", w->outputs, w->inputs);
    hipLaunchKernelGGL(w8_pack_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, codes, scales, static_cast<int8_t *>(packed), w->outputs, w->inputs,
                       w->chunks, blocks);
    return check_launch("w8_pack");
}

int32_t launch_w8(W8Args &a, int y, void *stream)
{
    switch (y) {
    case 0: return by_tokens<0>(a, stream);
    case 1 + SLORA_F16: return by_tokens<1 + SLORA_F16>(a, stream);
    }
    return by_tokens<1 + SLORA_BF16>(a, stream);
}

} // namespace slora
