// Operators on whole rows - norms around a block, rows in 8 bits: what the host side (rows.cpp) and the kernels (rows_kernels.hip) share.
#pragma once

#include "slora_internal.hpp"

struct slora_norm {
    int32_t width = 0, dtype = 0, flags = 0;
    float eps = 0, scale = 0;
    int device = -1;
    const uint16_t *post_weight = nullptr, *post_bias = nullptr, *pre_weight = nullptr, *pre_bias = nullptr;
};

namespace slora {

// the least largest magnitude that a row's codes are taken against: quotients with it are normal numbers
constexpr float kW8Least = 0x1p-100f;

// Rows are taken in pieces of eight elements.
constexpr int kPiece = 8;
constexpr int kRowThreads = 1024; // most of a workgroup

struct RowsOut {
    uint16_t *x; // 16 bits; NULL: not wanted
    int64_t x_stride;
    int8_t *codes; // 8 bits; NULL: not wanted
    int64_t codes_stride;
    float *scales;
};

struct NormArgs {
    const void *h;
    const uint16_t *block, *gate;
    void *h_out;
    int64_t h_stride, block_stride, gate_stride, h_out_stride;
    const uint16_t *post_weight, *post_bias, *pre_weight, *pre_bias;
    RowsOut out;
    float eps, scale;
    int32_t T, width;
    int32_t post, layer;
};

struct QuantizeArgs {
    const uint16_t *x, *gate;
    int64_t x_stride, gate_stride;
    RowsOut out;
    int32_t T, width, act;
};

// rows_kernels.hip
int32_t launch_norm(const NormArgs &a, int32_t dtype, bool h32, void *stream);
int32_t launch_quantize(const QuantizeArgs &a, int32_t dtype, void *stream);

} // namespace slora
