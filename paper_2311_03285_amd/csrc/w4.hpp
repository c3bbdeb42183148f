// Products with 4-bit weights: what the host side (w4.cpp) and the kernels (w4_kernels.hip) share.
#pragma once

#include "slora_internal.hpp"

// Packed matrix.  Tiles of 16 outputs x chunks of 128 inputs, 1 KiB each: lane l = 16 g + r of a wavefront has 16 bytes, word s of
// them the codes of output r and inputs 32 s + 8 g + i of the chunk, i = 0 .. 3 in the low halves of the four bytes and 4 .. 7 in the high ones.
// Behind them the scales, 16 per tile, chunk and unit of 32, 64 or 128 inputs (the largest of these that divides
// the group), then the zeros, one byte 0x80 | z each.  Outputs and inputs beyond the matrix have scale 0.
constexpr int kW4Rows = 16, kW4Chunk = 128;

struct slora_w4 {
    int32_t outputs = 0, inputs = 0, group = 0, dtype = 0;
    int32_t tiles = 0, chunks = 0, unit = 0;
    bool has_zeros = false;
    int device = -1;
    const uint8_t *packed = nullptr;
    int64_t code_bytes() const { return (int64_t)tiles * chunks * 1024; }
    int64_t units() const { return (int64_t)tiles * chunks * (kW4Chunk / unit) * kW4Rows; }
};

namespace slora {

struct W4Matrix {
    const uint8_t *codes;
    const uint16_t *scales;
    const uint8_t *zeros;
    const uint16_t *x;
    void *y;
    int32_t outputs, inputs, chunks;
    int32_t first; // workgroups of the matrices before
};
struct W4Args {
    W4Matrix m[SLORA_MAX_MULTI];
    int32_t n, T;
};

// w4_kernels.hip
int32_t launch_w4_pack(const slora_w4 *w, const void *codes, const void *scales, const uint8_t *zeros, void *packed, void *stream);
int32_t launch_w4(const slora_w4 *const *w, W4Args &a, bool y16, void *stream);

} // namespace slora
