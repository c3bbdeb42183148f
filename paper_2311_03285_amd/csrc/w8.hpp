// Products with 8-bit weights: what the host side (w8.cpp) and the kernels (w8_kernels.hip) share.
#pragma once

#include "slora_internal.hpp"

// Packed matrix.  Tiles of 16 outputs x chunks of 64 inputs, 1 KiB each: lane l = 16 g + r of a wavefront has 16 bytes, the codes of output r
// and inputs 16 g .. 16 g + 15 of the chunk.  Chunks come in pairs, outputs and inputs beyond the matrix have codes 0.  Behind them the scales, 16 per tile.
constexpr int kW8Rows = 16, kW8Chunk = 64, kW8Block = kW8Rows * kW8Chunk;

struct slora_w8 {
    int32_t outputs = 0, inputs = 0, dtype = 0;
    int32_t tiles = 0, chunks = 0;
    int device = -1;
    const int8_t *packed = nullptr;
    int64_t code_bytes() const { return (int64_t)tiles * chunks * kW8Block; }
    const float *scales() const { return reinterpret_cast<const float *>(packed + code_bytes()); }
};

namespace slora {

constexpr int64_t kW8MostStride = int64_t(1) << 22; // of rows of x, so that offsets in a workgroup's rows are 32 bits

struct W8Matrix {
    const int8_t *codes, *x;
    const float *scales, *x_scales;
    void *y;
    int64_t y_stride;
    int32_t outputs, chunks, tiles;
    int32_t x_stride, x_last; // x_last: where the last 16 bytes of a row begin
    int32_t first;            // workgroups of the matrices before
};
struct W8Args {
    W8Matrix m[SLORA_MAX_MULTI];
    int32_t n, T;
};

// How calls of more than 16 tokens are cut into workgroups
struct W8Shape {
    int outputs, tokens, threads;
    float us; // of a stage of 128 inputs
};
constexpr W8Shape kW8Shapes[] = {{256, 256, 512, 1.7f}, {256, 192, 512, 1.27f}, {256, 128, 512, 0.95f}, {128, 192, 512, 0.74f}, {128, 128, 256, 0.56f},
                                 {64, 128, 512, 0.42f}, {64, 64, 512, 0.3f},    {64, 32, 256, 0.2f},    {32, 32, 256, 0.18f}};
constexpr int64_t kComputeUnits = 256;
constexpr int64_t kOnceWeights = 64 << 20; // bytes
constexpr int64_t kMostThreads = (int64_t(1) << 32) - 1; // of a grid
inline int64_t w8_rounds(int64_t groups) { return (groups + kComputeUnits - 1) / kComputeUnits; }

// w8.cpp
int64_t w8_parts(const W8Args &a, int each); // how many of `each` outputs there are
int w8_shape(const W8Args &a);               // of kW8Shapes
bool w8_once(const W8Args &a, const W8Shape &s); // whether its weights are loaded without a place in the caches

// w8_kernels.hip
int32_t launch_w8_pack(const slora_w8 *w, const int8_t *codes, const float *scales, void *packed, void *stream);
// y: 0 fp32, else 1 + the 16-bit type
int32_t launch_w8(W8Args &a, int y, void *stream);

} // namespace slora
