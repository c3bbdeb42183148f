// Products with 8-bit weights: checks of the arguments.
#include <hip/hip_runtime_api.h>

#include <new>

#include "w8.hpp"

using namespace slora;

namespace slora {

int64_t w8_parts(const W8Args &a, int each)
{
    int64_t n = 0;
    for (int32_t k = 0; k < a.n; ++k) n += ((int64_t)a.m[k].outputs + each - 1) / each;
    return n;
}

// The shape whose workgroups, of which compute units take rounds, are done first, by what a stage of one takes (measured with one and with
// several rounds, where clocks are lower).  The larger the shape, the less is read for each product; the smaller, the more compute units have one.
// us: 256 x 256 against the next ones, 8192 tokens of 8192 x 8192 453 / 500 / 519, two of 20480 of 5120, 2048 tokens 387 / 418 / 441; 256 x 192 / 256 x 256, 5120 of
// 20480, 2048 tokens 197 / 211; 256 x 128 / 128 x 128, three of 4096 of 4096, 512 tokens 34 / 37; 128 x 192 / 128 x 128, three of 5003 of 3083, 333 tokens 33 / 42;
// 128 x 128 / 256 x 128, 4096 of 4096, 1024 tokens 25 / 30; 64 x 128 / 128 x 128, 512 tokens 17 / 22; 64 x 64 / 64 x 128, 200 tokens 13 / 15; 64 x 32 / 64 x 64, three,
// 24 tokens 14.5 / 15.0; 32 x 32 / 64 x 32, 64 tokens 8.8 / 11.9.  Teams: 64 x 64 with two 12.6, with one 17.8 (4096 of 4096, 64 tokens).
int w8_shape(const W8Args &a)
{
    int best = 0;
    float least = 0.0f;
    for (int i = 0; i < (int)(sizeof(kW8Shapes) / sizeof(kW8Shapes[0])); ++i) {
        const int64_t groups = w8_parts(a, kW8Shapes[i].outputs) * (((int64_t)a.T + kW8Shapes[i].tokens - 1) / kW8Shapes[i].tokens);
        const float us = (float)w8_rounds(groups) * kW8Shapes[i].us;
        if (i == 0 || (us < least && groups * kW8Shapes[i].threads <= kMostThreads)) {
            best = i;
            least = us;
        }
    }
    return best;
}

// Weights that are large, and that each are read by one workgroup or by several that run at the same time; with more rounds of workgroups the next tile of tokens finds in the memory-side cache
// what keeps its place.  us with / without a place, weights that are in no cache before: one tile of tokens, two of 20480 of 5120, 32 tokens 43.1 / 39.6, 100 tokens 49.3 / 46.9, four of 4096 of
// 4096, 128 tokens 23.6 / 20.4; one round, four of 4096 of 4096, 512 tokens 41.2 / 40.1, 8192 of 8192, 200 tokens 29.9 / 28.6, but 5120 of 20480, 300 tokens 58.5 / 62.8; more rounds, two of 20480 of
// 5120, 200 tokens 78 / 92, 900 tokens 227 / 273.  The largest two shapes read them at the same speed either way.
// Smaller weights gain less or lose, if they are still there: three of 4096 of 4096, 24 tokens, 14.2 / 13.5 from memory, 11.6 / 13.0 where all the weights that take turns are 200 MB.
bool w8_once(const W8Args &a, const W8Shape &s)
{
    int64_t bytes = 0;
    for (int32_t k = 0; k < a.n; ++k) bytes += (int64_t)a.m[k].tiles * a.m[k].chunks * kW8Block;
    const int64_t tiles = ((int64_t)a.T + s.tokens - 1) / s.tokens;
    return bytes >= kOnceWeights && (tiles == 1 || w8_rounds(w8_parts(a, s.outputs) * tiles) == 1);
}

} // namespace slora

namespace {

int32_t check_shape(int32_t outputs, int32_t inputs)
{
    if (outputs < 1 || outputs > 1 << 24) return fail(SLORA_EINVAL, "outputs=%d must be in [1, 2^24]", outputs);
    if (inputs < 1 || inputs > SLORA_W8_MAX_INPUTS) return fail(SLORA_EINVAL, "inputs=%d must be in [1, %d]", inputs, SLORA_W8_MAX_INPUTS);
    return SLORA_OK;
}

void shape(slora_w8 &w, int32_t outputs, int32_t inputs)
{
    w.outputs = outputs;
    w.inputs = inputs;
    w.tiles = (outputs + kW8Rows - 1) / kW8Rows;
    w.chunks = (inputs + 2 * kW8Chunk - 1) / (2 * kW8Chunk) * 2;
}

} // namespace

extern "C" {

int32_t slora_w8_bytes(int32_t outputs, int32_t inputs, int64_t *out)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    int32_t rc = check_shape(outputs, inputs);
    if (rc != SLORA_OK) return rc;
    slora_w8 w;
    shape(w, outputs, inputs);
    *out = w.code_bytes() + (int64_t)w.tiles * kW8Rows * 4;
    return SLORA_OK;
}

int32_t slora_w8_pack(slora_w8 **out, int32_t outputs, int32_t inputs, int32_t dtype, const int8_t *codes, const float *scales, void *packed,
                      void *stream)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    *out = nullptr;
    int32_t rc = check_shape(outputs, inputs);
    if (rc != SLORA_OK) return rc;
    if (dtype != SLORA_F16 && dtype != SLORA_BF16) return fail(SLORA_EINVAL, "unknown dtype %d", dtype);
    if (!codes || !scales || !packed) return fail(SLORA_EINVAL, "codes, scales and packed are needed");
    if (reinterpret_cast<uintptr_t>(packed) & 15) return fail(SLORA_EINVAL, "packed must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(scales) & 3) return fail(SLORA_EINVAL, "scales must be 4-byte aligned");
    slora_w8 *w = new (std::nothrow) slora_w8;
    if (!w) return fail(SLORA_ENOMEM, "out of host memory");
    shape(*w, outputs, inputs);
    w->dtype = dtype;
    w->packed = static_cast<const int8_t *>(packed);
    const hipError_t e = hipGetDevice(&w->device);
    rc = e == hipSuccess ? launch_w8_pack(w, codes, scales, packed, stream) : fail(SLORA_EHIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (rc != SLORA_OK) {
        delete w;
        return rc;
    }
    *out = w;
    return SLORA_OK;
}

int32_t slora_w8_destroy(slora_w8 *w)
{
    clear_error();
    delete w;
    return SLORA_OK;
}

} // extern "C"

namespace {
int32_t matmul(int32_t n, const slora_w8 *const *w, const int8_t *const *x, const int64_t *x_stride, const float *const *x_scales, int32_t T, void *const *y,
               const int64_t *y_stride, bool y16, void *stream)
{
    clear_error();
    if (n < 1 || n > SLORA_MAX_MULTI) return fail(SLORA_EINVAL, "n=%d must be in [1, %d]", n, SLORA_MAX_MULTI);
    if (!w || !x || !x_stride || !x_scales || !y || !y_stride) return fail(SLORA_EINVAL, "NULL argument");
    if (T < 0) return fail(SLORA_EINVAL, "T=%d is negative", T);
    if (T > 1 << 30) return fail(SLORA_ERANGE, "T=%d tokens are too many for one call", T); // (32-bit numbers of tokens, tiles' ends included)
    W8Args a{};
    a.n = n;
    a.T = T;
    for (int32_t k = 0; k < n; ++k) {
        if (!w[k]) return fail(SLORA_EINVAL, "w[%d] is NULL", k);
        if (w[k]->dtype != w[0]->dtype || w[k]->device != w[0]->device) return fail(SLORA_EINVAL, "w[%d] has another type or device than w[0]", k);
        if (T == 0) continue;
        if (!x[k] || !x_scales[k] || !y[k]) return fail(SLORA_EINVAL, "x[%d], x_scales[%d] or y[%d] is NULL", k, k, k);
        if ((reinterpret_cast<uintptr_t>(x[k]) | reinterpret_cast<uintptr_t>(y[k])) & 15) return fail(SLORA_EINVAL, "x[%d] and y[%d] must be 16-byte aligned", k, k);
        if (reinterpret_cast<uintptr_t>(x_scales[k]) & 3) return fail(SLORA_EINVAL, "x_scales[%d] must be 4-byte aligned", k);
        if (x_stride[k] < w[k]->inputs || x_stride[k] % 16 || x_stride[k] > kW8MostStride)
            return fail(SLORA_EINVAL, "x_stride[%d]=%lld must be a multiple of 16, at least %d and at most 2^22", k, (long long)x_stride[k], w[k]->inputs);
        if (y_stride[k] < w[k]->outputs || y_stride[k] > int64_t(1) << 29)
            return fail(SLORA_EINVAL, "y_stride[%d]=%lld must be at least %d and at most 2^29", k, (long long)y_stride[k], w[k]->outputs);
        for (int32_t m = 0; m < k; ++m)
            if (y[m] == y[k]) return fail(SLORA_EINVAL, "y[%d] and y[%d] are the same buffer", m, k);
        W8Matrix &to = a.m[k];
        to.codes = w[k]->packed;
        to.scales = w[k]->scales();
        to.x = x[k];
        to.x_scales = x_scales[k];
        to.y = y[k];
        to.y_stride = y_stride[k];
        to.outputs = w[k]->outputs;
        to.chunks = w[k]->chunks;
        to.tiles = w[k]->tiles;
        to.x_stride = (int32_t)x_stride[k];
        to.x_last = (w[k]->inputs - 1) / 16 * 16;
    }
    if (T == 0) return SLORA_OK;
    DeviceScope dev(w[0]->device);
    if (dev.status() != SLORA_OK) return dev.status();
    return launch_w8(a, y16 ? 1 + w[0]->dtype : 0, stream);
}
} // namespace

extern "C" {

int32_t slora_w8_matmul(int32_t n, const slora_w8 *const *w, const int8_t *const *x, const int64_t *x_stride, const float *const *x_scales, int32_t T,
                        float *const *y, const int64_t *y_stride, void *stream)
{
    return matmul(n, w, x, x_stride, x_scales, T, reinterpret_cast<void *const *>(y), y_stride, false, stream);
}

int32_t slora_w8_matmul_y16(int32_t n, const slora_w8 *const *w, const int8_t *const *x, const int64_t *x_stride, const float *const *x_scales, int32_t T,
                            void *const *y, const int64_t *y_stride, void *stream)
{
    return matmul(n, w, x, x_stride, x_scales, T, y, y_stride, true, stream);
}

} // extern "C"
