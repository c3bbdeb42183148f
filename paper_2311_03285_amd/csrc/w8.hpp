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

// w8_kernels.hip
int32_t launch_w8_pack(const slora_w8 *w, const int8_t *codes, const float *scales, void *packed, void *stream);
// y: 0 fp32, else 1 + the 16-bit type
int32_t launch_w8(W8Args &a, int y, void *stream);

} // namespace slora
