// Products with 4-bit weights: checks of the arguments.
#include <hip/hip_runtime_api.h>

#include <new>

#include "w4.hpp"

using namespace slora;

namespace {

int32_t check_shape(int32_t outputs, int32_t inputs, int32_t group)
{
    if (outputs < 1 || outputs > 1 << 24) return fail(SLORA_EINVAL, "outputs=%d must be in [1, 2^24]", outputs);
    if (inputs < 8 || inputs > 1 << 24 || inputs % 8) return fail(SLORA_EINVAL, "inputs=%d must be a multiple of 8 in [8, 2^24]", inputs);
    if (group < 32 || group % 32) return fail(SLORA_EINVAL, "group=%d must be a multiple of 32", group);
    return SLORA_OK;
}

void shape(slora_w4 &w, int32_t outputs, int32_t inputs, int32_t group)
{
    w.outputs = outputs;
    w.inputs = inputs;
    w.group = group;
    w.tiles = (outputs + kW4Rows - 1) / kW4Rows;
    w.chunks = (inputs + kW4Chunk - 1) / kW4Chunk;
    w.unit = group % 128 == 0 ? 128 : group % 64 == 0 ? 64 : 32;
}

} // namespace

extern "C" {

int32_t slora_w4_bytes(int32_t outputs, int32_t inputs, int32_t group, int64_t *out)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    int32_t rc = check_shape(outputs, inputs, group);
    if (rc != SLORA_OK) return rc;
    slora_w4 w;
    shape(w, outputs, inputs, group);
    *out = w.code_bytes() + 3 * w.units();
    return SLORA_OK;
}

int32_t slora_w4_pack(slora_w4 **out, int32_t outputs, int32_t inputs, int32_t group, int32_t dtype, const void *codes, const void *scales,
                      const uint8_t *zeros, void *packed, void *stream)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    *out = nullptr;
    int32_t rc = check_shape(outputs, inputs, group);
    if (rc != SLORA_OK) return rc;
    if (dtype != SLORA_F16 && dtype != SLORA_BF16) return fail(SLORA_EINVAL, "unknown dtype %d", dtype);
    if (!codes || !scales || !packed) return fail(SLORA_EINVAL, "codes, scales and packed are needed");
    if (reinterpret_cast<uintptr_t>(packed) & 15) return fail(SLORA_EINVAL, "packed must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(codes) & 3) return fail(SLORA_EINVAL, "codes must be 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(scales) & 1) return fail(SLORA_EINVAL, "scales must be 2-byte aligned");
    slora_w4 *w = new (std::nothrow) slora_w4;
    if (!w) return fail(SLORA_ENOMEM, "out of host memory");
    shape(*w, outputs, inputs, group);
    w->dtype = dtype;
    w->has_zeros = zeros != nullptr;
    w->packed = static_cast<const uint8_t *>(packed);
    const hipError_t e = hipGetDevice(&w->device);
    rc = e == hipSuccess ? launch_w4_pack(w, codes, scales, zeros, packed, stream) : fail(SLORA_EHIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (rc != SLORA_OK) {
        delete w;
        return rc;
    }
    *out = w;
    return SLORA_OK;
}

int32_t slora_w4_destroy(slora_w4 *w)
{
    clear_error();
    delete w;
    return SLORA_OK;
}

namespace {
int32_t matmul(int32_t n, const slora_w4 *const *w, const void *const *x, int32_t T, void *const *y, bool y16, void *stream)
{
    clear_error();
    if (n < 1 || n > SLORA_MAX_MULTI) return fail(SLORA_EINVAL, "n=%d must be in [1, %d]", n, SLORA_MAX_MULTI);
    if (!w || !x || !y) return fail(SLORA_EINVAL, "NULL argument");
    if (T < 0) return fail(SLORA_EINVAL, "T=%d is negative", T);
    W4Args a{};
    a.n = n;
    a.T = T;
    for (int32_t k = 0; k < n; ++k) {
        if (!w[k]) return fail(SLORA_EINVAL, "w[%d] is NULL", k);
        if (w[k]->dtype != w[0]->dtype || w[k]->group != w[0]->group || w[k]->device != w[0]->device)
            return fail(SLORA_EINVAL, "w[%d] has another type, group size or device than w[0]", k);
        if (T == 0) continue;
        if (!x[k] || !y[k]) return fail(SLORA_EINVAL, "x[%d] or y[%d] is NULL", k, k);
        if ((reinterpret_cast<uintptr_t>(x[k]) | reinterpret_cast<uintptr_t>(y[k])) & 15) return fail(SLORA_EINVAL, "x[%d] and y[%d] must be 16-byte aligned", k, k);
        for (int32_t m = 0; m < k; ++m)
            if (y[m] == y[k]) return fail(SLORA_EINVAL, "y[%d] and y[%d] are the same buffer", m, k);
        a.m[k].codes = w[k]->packed;
        a.m[k].scales = reinterpret_cast<const uint16_t *>(w[k]->packed + w[k]->code_bytes());
        a.m[k].zeros = w[k]->packed + w[k]->code_bytes() + 2 * w[k]->units();
        a.m[k].x = static_cast<const uint16_t *>(x[k]);
        a.m[k].y = y[k];
        a.m[k].outputs = w[k]->outputs;
        a.m[k].inputs = w[k]->inputs;
        a.m[k].chunks = w[k]->chunks;
    }
    if (T == 0) return SLORA_OK;
    DeviceScope dev(w[0]->device);
    if (dev.status() != SLORA_OK) return dev.status();
    return launch_w4(w, a, y16, stream);
}
} // namespace

int32_t slora_w4_matmul(int32_t n, const slora_w4 *const *w, const void *const *x, int32_t T, float *const *y, void *stream)
{
    return matmul(n, w, x, T, reinterpret_cast<void *const *>(y), false, stream);
}

int32_t slora_w4_matmul_y16(int32_t n, const slora_w4 *const *w, const void *const *x, int32_t T, void *const *y, void *stream)
{
    return matmul(n, w, x, T, y, true, stream);
}

} // extern "C"
