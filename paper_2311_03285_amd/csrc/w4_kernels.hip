// gfx950 kernels of the products with 4-bit weights: packing, and y = x W for a few tokens.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

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

constexpr int kWave = 64;
constexpr int kWaves = 8; // of a workgroup: they share out the chunks of its outputs' inputs

template <int DT>
__device__ __forceinline__ float widen(uint16_t b)
{
    return DT == SLORA_F16 ? (float)__builtin_bit_cast(_Float16, b) : __uint_as_float((uint32_t)b << 16);
}
template <int DT>
__device__ __forceinline__ uint16_t narrow(float f)
{
    if constexpr (DT == SLORA_F16)
        return __builtin_bit_cast(uint16_t, (_Float16)f);
    else
        return __builtin_bit_cast(uint16_t, (__bf16)f);
}

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
        if (zeros) packed[code_bytes + 2 * units + at] = in ? zeros[from] : (uint8_t)0;
    }
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
// Matrix instruction 16 x 16 x 32: outputs are rows, tokens columns; lane l = 16 g + n supplies inputs 8 g .. 8 g + 7 of row or column n,
// and receives rows 4 g .. 4 g + 3 of column n.
//
// The bits of a code c = 0 .. 15, taken as an 8-bit float of four exponent and three mantissa bits (bias 7), are the
// number c * 2^-9 - the least exponent's numbers and the subnormal ones go up in even steps - so that one conversion of two bytes makes two operands,
// exact in either 16-bit type.  A unit's products are summed as c * 2^-9 * x; the zero is taken off as z times the sum of
// x, which a matrix of ones in a further instruction gives every lane for its column.
template <int DT>
struct Operand;
template <>
struct Operand<SLORA_F16> {
    typedef f16x8 type;
    static __device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f16x8 codes(uint32_t u)
    {
        const uint32_t lo = u & 0x0f0f0f0fu, hi = (u >> 4) & 0x0f0f0f0fu;
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
        return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
    }
};
template <>
struct Operand<SLORA_BF16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ bf16x8 codes(uint32_t u)
    {
        const uint32_t lo = u & 0x0f0f0f0fu, hi = (u >> 4) & 0x0f0f0f0fu;
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// A workgroup = RT tiles of 16 outputs x NT of 16 tokens; its wavefronts take chunks of 128 inputs in turn and are added in LDS.
template <int DT, int RT, int NT, int U>
__global__ __launch_bounds__(kWaves *kWave) void w4_kernel(W4Args a, bool y16)
{
    typedef typename Operand<DT>::type operand;
    constexpr int kPer = kW4Chunk / U; // units of a chunk
    __shared__ float part[kWaves][RT * 16][NT * 16 + 1];
    int k = 0;
    while (k + 1 < a.n && (int)blockIdx.x >= a.m[k + 1].first) ++k;
    const W4Matrix &m = a.m[k];
    const int tiles = (m.outputs + kW4Rows - 1) / kW4Rows;
    const int tile0 = ((int)blockIdx.x - m.first) * RT, t0 = blockIdx.y * (NT * 16);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;

    operand one;
#pragma unroll
    for (int i = 0; i < 8; ++i) one[i] = 1.0f;
    f32x4 sum[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int c = wave; c < m.chunks; c += kWaves) {
        u32x4 w[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) // (tiles beyond the last: the last once more, whose sums nobody takes)
            w[r] = *reinterpret_cast<const u32x4 *>(m.codes + ((int64_t)min(tile0 + r, tiles - 1) * m.chunks + c) * 1024 + lane * 16);
        u32x4 x[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int token = t0 + t * 16 + n, at = c * kW4Chunk + s * 32 + g * 8;
                x[t][s] = token < a.T && at < m.inputs ? *reinterpret_cast<const u32x4 *>(m.x + (int64_t)token * m.inputs + at) : u32x4{0u, 0u, 0u, 0u};
            }
        f32x4 ones[kPer][NT];
#pragma unroll
        for (int u = 0; u < kPer; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                ones[u][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = u * (U / 32); s < (u + 1) * (U / 32); ++s) ones[u][t] = Operand<DT>::mfma(one, __builtin_bit_cast(operand, x[t][s]), ones[u][t]);
            }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int64_t unit0 = ((int64_t)min(tile0 + r, tiles - 1) * m.chunks + c) * kPer * kW4Rows + 4 * g;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const u32x2 sc = *reinterpret_cast<const u32x2 *>(m.scales + unit0 + u * kW4Rows);
                const uint32_t z = m.zeros ? *reinterpret_cast<const uint32_t *>(m.zeros + unit0 + u * kW4Rows) : 0x08080808u;
                f32x4 acc[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = u * (U / 32); s < (u + 1) * (U / 32); ++s) {
                    const operand cw = Operand<DT>::codes(w[r][s]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = Operand<DT>::mfma(cw, __builtin_bit_cast(operand, x[t][s]), acc[t]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float scale = widen<DT>((uint16_t)(sc[i / 2] >> (16 * (i % 2)))), zero = (float)((z >> (8 * i)) & 255u);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        sum[r][t][i] = __builtin_fmaf(__builtin_fmaf(-zero, ones[u][t][i], 512.0f * acc[t][i]), scale, sum[r][t][i]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][r * 16 + 4 * g + i][t * 16 + n] = sum[r][t][i];
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 16 * NT * 16; i += kWaves * kWave) {
        const int row = i % (RT * 16), t = i / (RT * 16), o = tile0 * kW4Rows + row;
        if (o >= m.outputs || t0 + t >= a.T) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += part[w][row][t];
        const int64_t at = (int64_t)(t0 + t) * m.outputs + o;
        if (y16)
            static_cast<uint16_t *>(m.y)[at] = narrow<DT>(v);
        else
            static_cast<float *>(m.y)[at] = v;
    }
}

int32_t check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SLORA_OK : fail(SLORA_EHIP, "launching %s: %s", what, hipGetErrorString(e));
}

template <int DT, int RT, int NT, int U>
int32_t launch(W4Args &a, bool y16, void *stream)
{
    int64_t groups = 0;
    for (int32_t k = 0; k < a.n; ++k) {
        a.m[k].first = (int32_t)groups;
        groups += ((int64_t)a.m[k].outputs + kW4Rows * RT - 1) / (kW4Rows * RT);
    }
    const int64_t token_blocks = ((int64_t)a.T + NT * 16 - 1) / (NT * 16);
    if (groups > INT32_MAX || token_blocks > 65535) return fail(SLORA_ERANGE, "T=%d tokens are too many for one call", a.T);
    hipLaunchKernelGGL((w4_kernel<DT, RT, NT, U>), dim3((unsigned)groups, (unsigned)token_blocks), dim3(kWaves * kWave), 0, (hipStream_t)stream, a, y16);
    return check_launch("w4");
}

template <int DT, int U>
int32_t by_tokens(W4Args &a, bool y16, void *stream)
{
    if (a.T <= 16) return launch<DT, 1, 1, U>(a, y16, stream);
    if (a.T <= 32) return launch<DT, 1, 2, U>(a, y16, stream);
    return launch<DT, 1, 4, U>(a, y16, stream);
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
