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

// The sum, exact so far, is rounded to fp32 and multiplied by both scales there; the product of the scales alone could leave the range that the three have.  So could the
// sum, up to 2^31, times a scale of x above 2^96 (a row of bfloat16 has up to 2^121): of that, 2^32 wait until the end.  What is left is above 2^64, so that no weight's
// scale makes a subnormal number of it, and results are the same to the bit.
struct XScale {
    float now, rest;
    __device__ __forceinline__ explicit XScale(float s)
    {
        const bool far = fabsf(s) > 0x1p96f;
        now = far ? s * 0x1p-32f : s;
        rest = far ? 0x1p32f : 1.0f;
    }
};
// Y: 0 fp32, else 1 + the 16-bit type
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

// Up to 16 tokens: weights go from memory to the matrix instruction's registers.  A workgroup = RT tiles of 16 outputs; its wavefronts take chunks of inputs
// in turn and are added up in LDS.
// Weights of any size are loaded without a place in the caches: of a model whose layers take turns they are never there.  us with / without a place: 16 tokens, two of 20480 of 5120,
// weights that are in no cache 43.9 / 39.8, three of 4096 of 4096 13.5 / 12.7; where all the weights that take turns are 200 MB 31.4 / 38.7 and 10.2 / 12.3.
// Bound: HBM and the time to fill it: four of 4096 of 4096, one token 12.4 us from memory = 5.4 TB/s, 11.4 where 200 MB of them take turns; two of 20480 of 5120, one token 32 us = 6.5 TB/s, 16 tokens 39 us.  With more
// tokens every 16 outputs read all of x again: two of 20480 of 5120, 32 tokens 81 us with one tile, 55 with two, 42 from LDS below.
constexpr int kFewWaves = 8, kFewTokens = 16;
template <int RT, int Y>
__global__ __launch_bounds__(kFewWaves *kWave) void w8_few_kernel(W8Args a)
{
    constexpr int kAhead = 4; // chunks under way
    __shared__ int part[kFewWaves][RT][4][kWave];
    const W8Matrix &m = a.m[matrix_of(a, blockIdx.x)];
    const int wave = wave_number(), lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    const int tile0 = ((int)blockIdx.x - m.first) * RT, chunks = m.chunks, x_last = m.x_last;

    i32x4 sum[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = i32x4{0, 0, 0, 0};
    // (tokens behind the last: the last once more, whose sums nobody takes)
    const int8_t *const row = m.x + (int64_t)min(n, a.T - 1) * m.x_stride, *codes[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) codes[r] = m.codes + (int64_t)min(tile0 + r, m.tiles - 1) * chunks * kW8Block + lane * 16;

    struct Chunk {
        i32x4 w[RT], x;
    } ring[kAhead];
    // (inputs behind the last: weights of 0)
    auto fetch = [&](Chunk &to, int c) {
#pragma unroll
        for (int r = 0; r < RT; ++r) to.w[r] = __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(codes[r] + (int64_t)c * kW8Block));
        to.x = *reinterpret_cast<const i32x4 *>(row + min(c * kW8Chunk + g * 16, x_last));
    };
    auto work = [&](const Chunk &now) {
#pragma unroll
        for (int r = 0; r < RT; ++r) sum[r] = mfma16(now.x, now.w[r], sum[r]);
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
    // token 4 g + i of output n is register i
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][r][i][lane] = sum[r][i];
    __syncthreads();
    for (int w = threadIdx.x; w < RT * kW8Rows * a.T; w += kFewWaves * kWave) {
        const int r = w % (RT * kW8Rows), t = w / (RT * kW8Rows), o = tile0 * kW8Rows + r;
        if (o >= m.outputs) continue;
        int total = 0;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) total += part[k][r / 16][t % 4][t / 4 * 16 + r % 16];
        const XScale by(m.x_scales[t]);
        store_y<Y>(m.y, (int64_t)t * m.y_stride + o, (float)total * by.now * m.scales[o] * by.rest);
    }
}

// Many tokens: a workgroup takes WO * MO * 32 outputs and WT * MT * 32 tokens, WO x WT wavefronts of them, in stages of 128 inputs that go through LDS: two
// buffers, one that is read while the next stage is written to the other, whose bytes have come from memory a stage before.
// Where that gives few workgroups, TEAMS of such wavefronts take stages in turn, each through buffers of its own, and are added up at the end.
// LDS holds units of 16 bytes, [16 rows][chunk of 64][piece of 16][row]: an operand's read is 16 lanes of neighbouring units.  Weights lie so in memory.
// Rows of x come in eights of pieces (128 bytes); a row's place among 16 is permuted by the piece's number, so that the lanes that write
// eights or sixteens of pieces are in different banks.
// Outputs are the rows of the matrix instruction here, so that a lane has four neighbouring ones of a token, which go to LDS together and from there
// to y in rows.
// Bound, large products: power.  8192 tokens of 8192 x 8192 439 - 476 us by the card = 2310 - 2500 TOP/s; the matrix units are busy for 74 % of the cycles, at 1.5 GHz of
// 2.4.  (1676 TOP/s with operands read right before they are used and y stored from registers, 2120 with reads spread in groups and y through LDS, 2323 with
// one read, write or load behind each product, 2420 with two wavefronts a SIMD instead of one.)  Small ones: the stages' chain of barrier, LDS and product; 512
// tokens of 4096 x 4096 17 us, of which products at that rate take 8.  Between 17 and 100 tokens the weights' bytes: two of 20480 of 5120, 32 tokens 38 us = 5.6 TB/s.
constexpr int kStageBytes = 2 * kW8Chunk;
constexpr int kRaw = 0x00027000; // a buffer of 32-bit words, without a format
// ONCE: weights are loaded without a place in the caches (bit 1 of a load's last argument).
constexpr int kNowhere = 1 << 30; // an offset behind every buffer's end: loads are 0

template <int TEAMS, int WO, int WT, int MO, int MT>
struct Tile {
    static constexpr int kTeam = WO * WT * kWave, kThreads = TEAMS * kTeam; // threads
    static constexpr int BO = WO * MO * 32, BT = WT * MT * 32, kUnits = 8;  // units of a row and stage
    static constexpr int kStages = 2 * (BO + BT) * kUnits;                  // of a team
    static constexpr int kWaves = kThreads / kWave;
    static constexpr int lds(int y_bytes) // stages, or all teams' sums but one's, or the outputs of 32 tokens of each wavefront
    {
        const int pitch = MO * 32 * y_bytes + 16;
        return std::max({TEAMS * kStages * 16, (TEAMS - 1) * kTeam * MO * MT * 64, WO * WT * 32 * pitch});
    }
};
// wavefronts of a SIMD that registers are kept for: with 128 sums a lane (256 x 256) one, which leaves room for two all the same (234 registers)
constexpr int tile_occupancy(int blocks) { return blocks >= 8 ? 1 : 2; }

template <int TEAMS, int WO, int WT, int MO, int MT, bool ONCE, int Y>
__global__ __launch_bounds__(TEAMS *WO *WT *kWave, tile_occupancy(MO *MT)) void w8_tile_kernel(W8Args a)
{
    typedef Tile<TEAMS, WO, WT, MO, MT> Shape;
    constexpr int BO = Shape::BO, BT = Shape::BT, kUnits = Shape::kUnits, kTeam = Shape::kTeam;
    constexpr int kPutsX = BT * kUnits / kTeam, kPutsW = BO * kUnits / kTeam, kPuts = kPutsX + kPutsW; // units of a thread and stage
    constexpr int kReads = MT + MO;
    extern __shared__ i32x4 lds[]; // [team] {[2][BT * kUnits], [2][BO * kUnits]}
    const int k = matrix_of(a, blockIdx.x);
    const W8Matrix &m = a.m[k];
    const int wave = wave_number() % (WO * WT), team = wave_number() / (WO * WT), thread = threadIdx.x % kTeam, lane = threadIdx.x % kWave, n = lane % 32, h = lane / 32;
    const int wt = wave / WO, wo = wave % WO;
    i32x4 *const lds_x = lds + team * Shape::kStages, *const lds_w = lds_x + 2 * BT * kUnits;

    // (Giving each die a run of neighbouring tiles was no faster: 8192 tokens of 8192 x 8192 464 - 468 us either way, 5376 of 5120 237 / 243.)
    const int tiles_o = (m.outputs + BO - 1) / BO, block = (int)blockIdx.x - m.first;
    const int t0 = block / tiles_o * BT, o0 = block % tiles_o * BO;

    // This thread's units of a stage: of x, number thread % 8 of rows thread / 8 and on; of the weights, number thread and on.  Where a row or the last
    // tile ends inside a stage, loads go on into what is behind, whose weights are 0, as far as the rows of the workgroup, or the codes, reach; loads beyond are 0.
    const int stages = m.chunks / 2, rows = min(BT, a.T - t0), tiles = min(BO / kW8Rows, m.tiles - o0 / kW8Rows);
    const auto x_rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(m.x + (int64_t)t0 * m.x_stride), 0, (rows - 1) * m.x_stride + m.x_last + 16, kRaw);
    const auto w_tiles = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(m.codes + (int64_t)(o0 / kW8Rows) * m.chunks * kW8Block), 0, tiles * m.chunks * kW8Block, kRaw);
    const int piece = thread % 8, row0 = thread / 8;
    auto place = [](int p) { return 2 * p ^ p / 4; }; // permutes the rows of a piece
    const auto x_put = [&](int j) { // (constant steps of j where a team has 16 rows of threads or more)
        const int row = row0 + j * (kTeam / 8);
        return (row / 16 * 2 + piece / 4) * 64 + piece % 4 * 16 + ((row % 16) ^ place(piece));
    };
    int at[kPuts];
#pragma unroll
    for (int j = 0; j < kPutsX; ++j) at[j] = min(row0 + j * (kTeam / 8), rows - 1) * m.x_stride + piece * 16;
#pragma unroll
    for (int j = 0; j < kPutsW; ++j) {
        const int u = thread + j * kTeam;
        at[kPutsX + j] = min(u / 128, tiles - 1) * m.chunks * kW8Block + u % 128 * 16;
    }
    i32x4 raw[kPuts];
    auto fetch = [&](int j, int s) { // turn s of this team

        const int number = s * TEAMS + team;
        if (j < kPutsX)
            raw[j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(x_rows, at[j] + (number < stages ? number * kStageBytes : kNowhere), 0, 0));
        else
            raw[j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_tiles, at[j] + (number < stages ? number * (2 * kW8Block) : kNowhere), 0, ONCE ? 2 : 0));
    };
    auto put = [&](int j, int buffer) {
        if (j < kPutsX)
            lds_x[buffer * BT * kUnits + x_put(j)] = raw[j];
        else
            lds_w[buffer * BO * kUnits + thread + (j - kPutsX) * kTeam] = raw[j];
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

    // Operands are read a step ahead, and a quarter of a stage's units is written in each step.  The buffer that step 3 leaves takes the first quarter of the stage after
    // next there, and the other ones in the steps that follow; registers that have been written take the stage after that.  (Behind the last stage: zeros.)
    // More of either, operands two steps and units two or three stages ahead, was no faster (512 tokens of 4096 x 4096, cold weights, 22 us each).
    auto quarter = [](int q) { return q * kPuts / 4; };
    const int turns = (stages + TEAMS - 1) / TEAMS;
#pragma unroll
    for (int j = 0; j < kPuts; ++j) fetch(j, 0);
#pragma unroll
    for (int j = 0; j < kPuts; ++j) {
        put(j, 0);
        fetch(j, 1);
    }
#pragma unroll
    for (int j = 0; j < quarter(1); ++j) {
        put(j, 1);
        fetch(j, 2);
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(i, 0, 0);
    for (int s = 0; s < turns; ++s) {
        const int buffer = s % 2;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const bool crosses = ks == 3;
            if (crosses) lds_barrier(); // the next stage is in the other buffer; nobody reads this one any more
            const int q = (ks + 1) % 4, beside = kReads + 2 * (quarter(q + 1) - quarter(q));
#pragma unroll
            for (int p = 0; p < MO * MT; ++p) {
                sum[p / MT][p % MT] = mfma32(wf[ks % 2][p / MT], xf[ks % 2][p % MT], sum[p / MT][p % MT]);
                // beside each product: operands first, then units to LDS and from memory in turn
#pragma unroll
                for (int o = p * beside / (MO * MT); o < (p + 1) * beside / (MO * MT); ++o) {
                    const int j = quarter(q) + (o - kReads) / 2;
                    if (o < kReads)
                        read(o, crosses ? buffer ^ 1 : buffer, q);
                    else if ((o - kReads) % 2 == 0)
                        put(j, crosses ? buffer : buffer ^ 1);
                    else
                        fetch(j, s + (crosses ? 3 : 2));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if constexpr (TEAMS > 1) { // the other teams' sums to the first
        lds_barrier();
        i32x4 *const merge = lds + (team - 1) * kTeam * MO * MT * 4 + thread;
        if (team > 0) {
#pragma unroll
            for (int i = 0; i < MO * MT; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const i32x16 &v = sum[i / MT][i % MT];
                    merge[(i * 4 + b) * kTeam] = i32x4{v[4 * b], v[4 * b + 1], v[4 * b + 2], v[4 * b + 3]};
                }
        }
        lds_barrier();
        if (team == 0) {
#pragma unroll
            for (int k = 1; k < TEAMS; ++k)
#pragma unroll
                for (int i = 0; i < MO * MT; ++i)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const i32x4 v = lds[(k - 1) * kTeam * MO * MT * 4 + thread + (i * 4 + b) * kTeam];
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[i / MT][i % MT][4 * b + e] += v[e];
                    }
        }
    }
    lds_barrier();
    if (team > 0) return;
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
        const XScale by(m.x_scales[min(tw + n, a.T - 1)]);
        const bool far = __builtin_amdgcn_ballot_w64(by.rest != 1.0f) != 0;
        auto put_y = [&](auto far) {
#pragma unroll
            for (int i = 0; i < MO; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const f32x4 w_scale = *reinterpret_cast<const f32x4 *>(m.scales + min(ow + i * 32 + 8 * b + 4 * h, m.tiles * kW8Rows - 4));
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (float)sum[i][j][4 * b + e] * by.now * w_scale[e];
                    if (far) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] *= by.rest;
                    }
                    char *const to = stage + n * kPitch + (i * 32 + 8 * b + 4 * h) * sizeof(Out);
                    if constexpr (Y == 0)
                        *reinterpret_cast<f32x4 *>(to) = f32x4{v[0], v[1], v[2], v[3]};
                    else
                        *reinterpret_cast<u32x2 *>(to) = u32x2{(uint32_t)narrow<Y - 1>(v[0]) | (uint32_t)narrow<Y - 1>(v[1]) << 16,
                                                               (uint32_t)narrow<Y - 1>(v[2]) | (uint32_t)narrow<Y - 1>(v[3]) << 16};
                }
        };
        // Scales far from 1 are asked for at every four outputs, or (twice the code) once.  us so / so: three of 5003 of 3083, 333 tokens 31.0 / 31.7; two of 16384 of 4096, 2048 tokens
        // (256 x 256) 267 / 264, of which 263 without asking.
        if constexpr (MO * MT < 6)
            put_y(far);
        else if (far)
            put_y(std::true_type{});
        else
            put_y(std::false_type{});
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
#pragma unroll 8
            for (int i = lane; i < 32 * MO * 32; i += kWave) {
                const int row = i / (MO * 32), e = i % (MO * 32);
                if (tw + row < a.T && ow + e < m.outputs) y[(int64_t)(tw + row) * m.y_stride + ow + e] = *reinterpret_cast<const Out *>(stage + row * kPitch + e * sizeof(Out));
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    }
}

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

template <int RT, int Y>
int32_t launch_few(W8Args &a, void *stream)
{
    const int64_t groups = share_out(a, RT * kW8Rows, 1);
    if (groups * kFewWaves * kWave > kMostThreads) return fail(SLORA_ERANGE, "the matrices have too many outputs for one call");
    hipLaunchKernelGGL((w8_few_kernel<RT, Y>), dim3((unsigned)groups), dim3(kFewWaves * kWave), 0, (hipStream_t)stream, a);
    return check_launch("w8_few");
}

template <int SHAPE, int TEAMS, int WO, int WT, int MO, int MT, bool ONCE, int Y>
int32_t launch_tile(W8Args &a, void *stream)
{
    typedef Tile<TEAMS, WO, WT, MO, MT> Shape;
    constexpr int kLds = Shape::lds(Y == 0 ? 4 : 2);
    static_assert(kLds <= 160 * 1024, "LDS");
    static_assert(kW8Shapes[SHAPE].outputs == Shape::BO && kW8Shapes[SHAPE].tokens == Shape::BT && kW8Shapes[SHAPE].threads == Shape::kThreads, "the shape that w8_shape has chosen");
    const int64_t groups = share_out(a, Shape::BO, ((int64_t)a.T + Shape::BT - 1) / Shape::BT);
    if (groups * Shape::kThreads > kMostThreads) return fail(SLORA_ERANGE, "T=%d tokens of so many outputs are too many for one call", a.T);
    if (kLds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&w8_tile_kernel<TEAMS, WO, WT, MO, MT, ONCE, Y>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return fail(SLORA_EHIP, "hipFuncSetAttribute(LDS size): %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL((w8_tile_kernel<TEAMS, WO, WT, MO, MT, ONCE, Y>), dim3((unsigned)groups), dim3(Shape::kThreads), kLds, (hipStream_t)stream, a);
    return check_launch("w8_tile");
}

// Up to 16 tokens: one tile of outputs a workgroup or two, by the bytes that the compute unit with most workgroups reads.  us with one / two: 16 tokens, two of 20480 of
// 5120 52 / 39, 5120 of 20480 37 / 28, 4096 of 4096 5.8 / 6.7; 8 tokens, three of 4096 of 4096 10.6 / 11.3.
template <int Y>
int32_t few(W8Args &a, void *stream)
{
    const int64_t tiles = w8_parts(a, kW8Rows);
    if (w8_rounds(tiles) * (16 + a.T) <= w8_rounds((tiles + 1) / 2) * (32 + a.T) && tiles * kFewWaves * kWave <= kMostThreads) return launch_few<1, Y>(a, stream);
    return launch_few<2, Y>(a, stream);
}

template <int Y>
int32_t many(W8Args &a, void *stream)
{
    const int shape = w8_shape(a);
    auto by_once = [&](auto launch) { return w8_once(a, kW8Shapes[shape]) ? launch(std::true_type{}) : launch(std::false_type{}); };
    switch (shape) {
    case 0: return launch_tile<0, 1, 2, 4, 4, 2, false, Y>(a, stream);
    case 1: return launch_tile<1, 1, 4, 2, 2, 3, false, Y>(a, stream);
    case 2: return by_once([&](auto once) { return launch_tile<2, 1, 4, 2, 2, 2, once.value, Y>(a, stream); });
    case 3: return by_once([&](auto once) { return launch_tile<3, 1, 4, 2, 1, 3, once.value, Y>(a, stream); });
    case 4: return by_once([&](auto once) { return launch_tile<4, 1, 2, 2, 2, 2, once.value, Y>(a, stream); });
    case 5: return by_once([&](auto once) { return launch_tile<5, 2, 2, 2, 1, 2, once.value, Y>(a, stream); });
    case 6: return by_once([&](auto once) { return launch_tile<6, 2, 2, 2, 1, 1, once.value, Y>(a, stream); });
    case 7: return by_once([&](auto once) { return launch_tile<7, 2, 2, 1, 1, 1, once.value, Y>(a, stream); });
    }
    return by_once([&](auto once) { return launch_tile<8, 4, 1, 1, 1, 1, once.value, Y>(a, stream); });
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
    auto by_tokens = [&](auto type) { return a.T <= kFewTokens ? few<type.value>(a, stream) : many<type.value>(a, stream); };
    switch (y) {
    case 0: return by_tokens(std::integral_constant<int, 0>{});
    case 1 + SLORA_F16: return by_tokens(std::integral_constant<int, 1 + SLORA_F16>{});
    }
    return by_tokens(std::integral_constant<int, 1 + SLORA_BF16>{});
}

} // namespace slora
