// Norms around a block and rows in 8 bits: checks of the arguments.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <new>

#include "rows.hpp"

using namespace slora;

namespace {

int32_t check_rows(const char *name, const void *p, int64_t stride, int32_t width, int32_t multiple)
{
    if (!p) return fail(SLORA_EINVAL, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & 15) return fail(SLORA_EINVAL, "%s must be 16-byte aligned", name);
    // (a stride that T rows of would pass 2^63 bytes is no stride)
    if (stride < width || stride % multiple || stride > int64_t(1) << 29)
        return fail(SLORA_EINVAL, "%s: stride %lld must be a multiple of %d, at least %d and at most 2^29", name, (long long)stride, multiple, width);
    return SLORA_OK;
}

// what may be left out, of rows that are
int32_t check_out(const RowsOut &o, const char *x_name, int32_t width)
{
    int32_t rc = SLORA_OK;
    if (o.x) rc = check_rows(x_name, o.x, o.x_stride, width, kPiece);
    if (rc == SLORA_OK && o.codes) rc = check_rows("codes", o.codes, o.codes_stride, width, 16);
    if (rc != SLORA_OK) return rc;
    if (!o.codes != !o.scales) return fail(SLORA_EINVAL, "codes and scales go together");
    if (reinterpret_cast<uintptr_t>(o.scales) & 3) return fail(SLORA_EINVAL, "scales must be 4-byte aligned");
    if (o.codes && (const void *)o.codes == (const void *)o.x) return fail(SLORA_EINVAL, "codes and %s are the same buffer", x_name);
    return SLORA_OK;
}

} // namespace

extern "C" {

int32_t slora_norm_init(slora_norm **out, int32_t width, int32_t dtype, int32_t flags, float eps, float scale, const void *post_weight,
                        const void *post_bias, const void *pre_weight, const void *pre_bias)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    *out = nullptr;
    if (width < 1 || width > SLORA_NORM_MAX_WIDTH) return fail(SLORA_EINVAL, "width=%d must be in [1, %d]", width, SLORA_NORM_MAX_WIDTH);
    if (dtype != SLORA_F16 && dtype != SLORA_BF16) return fail(SLORA_EINVAL, "unknown dtype %d", dtype);
    if (flags & ~(SLORA_NORM_LAYER | SLORA_NORM_POST | SLORA_NORM_H32)) return fail(SLORA_EINVAL, "unknown flags %d", flags);
    if (!std::isfinite(eps) || !(eps == 0.0f || eps >= 0x1p-60f)) return fail(SLORA_EINVAL, "eps=%g must be 0 or at least 2^-60", (double)eps);
    if (!std::isfinite(scale)) return fail(SLORA_EINVAL, "scale must be finite");
    if (!(flags & SLORA_NORM_POST) && (post_weight || post_bias)) return fail(SLORA_EINVAL, "post_weight and post_bias need SLORA_NORM_POST");
    const void *const vectors[] = {post_weight, post_bias, pre_weight, pre_bias};
    for (const void *v : vectors)
        if (reinterpret_cast<uintptr_t>(v) & 15) return fail(SLORA_EINVAL, "weights and biases must be 16-byte aligned");
    slora_norm *n = new (std::nothrow) slora_norm;
    if (!n) return fail(SLORA_ENOMEM, "out of host memory");
    n->width = width;
    n->dtype = dtype;
    n->flags = flags;
    n->eps = eps;
    n->scale = scale;
    n->post_weight = static_cast<const uint16_t *>(post_weight);
    n->post_bias = static_cast<const uint16_t *>(post_bias);
    n->pre_weight = static_cast<const uint16_t *>(pre_weight);
    n->pre_bias = static_cast<const uint16_t *>(pre_bias);
    const hipError_t e = hipGetDevice(&n->device);
    if (e != hipSuccess) {
        delete n;
        return fail(SLORA_EHIP, "hipGetDevice: %s", hipGetErrorString(e));
    }
    *out = n;
    return SLORA_OK;
}

int32_t slora_norm_destroy(slora_norm *norm)
{
    clear_error();
    delete norm;
    return SLORA_OK;
}

int32_t slora_norm_apply(const slora_norm *norm, int32_t T, const void *h, int64_t h_stride, const void *block, int64_t block_stride, const void *gate,
                         int64_t gate_stride, void *h_out, int64_t h_out_stride, void *x, int64_t x_stride, int8_t *codes, int64_t codes_stride,
                         float *scales, void *stream)
{
    clear_error();
    if (!norm) return fail(SLORA_EINVAL, "norm is NULL");
    if (T < 0) return fail(SLORA_EINVAL, "T=%d is negative", T);
    if (T == 0) return SLORA_OK;
    const int32_t n = norm->width;
    int32_t rc = check_rows("h", h, h_stride, n, kPiece);
    if (rc == SLORA_OK && block) rc = check_rows("block", block, block_stride, n, kPiece);
    if (rc == SLORA_OK && gate && gate_stride != 0) rc = check_rows("gate", gate, gate_stride, n, kPiece);
    if (rc == SLORA_OK && h_out) rc = check_rows("h_out", h_out, h_out_stride, n, kPiece);
    if (rc != SLORA_OK) return rc;
    if (gate && !block) return fail(SLORA_EINVAL, "a gate needs a block");
    if (reinterpret_cast<uintptr_t>(gate) & 15) return fail(SLORA_EINVAL, "gate must be 16-byte aligned");
    if (h_out == h && h_out_stride != h_stride) return fail(SLORA_EINVAL, "h_out is h with another stride");
    if (x && x == block && x_stride != block_stride) return fail(SLORA_EINVAL, "x is block with another stride");
    if (x && (x == h || x == h_out || x == gate)) return fail(SLORA_EINVAL, "x is the buffer of h, h_out or gate");
    if (h_out && (h_out == block || h_out == gate)) return fail(SLORA_EINVAL, "h_out is the buffer of block or gate");
    NormArgs a{};
    a.out = {static_cast<uint16_t *>(x), x_stride, codes, codes_stride, scales};
    if ((rc = check_out(a.out, "x", n)) != SLORA_OK) return rc;
    if (codes && (codes == h || codes == block || codes == gate || codes == h_out)) return fail(SLORA_EINVAL, "codes is another array's buffer");
    if (!h_out && !x && !codes) return fail(SLORA_EINVAL, "h_out, x or codes is needed");
    a.h = h;
    a.block = static_cast<const uint16_t *>(block);
    a.gate = static_cast<const uint16_t *>(gate);
    a.h_out = h_out;
    a.h_stride = h_stride;
    a.block_stride = block_stride;
    a.gate_stride = gate_stride;
    a.h_out_stride = h_out_stride;
    a.post_weight = norm->post_weight;
    a.post_bias = norm->post_bias;
    a.pre_weight = norm->pre_weight;
    a.pre_bias = norm->pre_bias;
    a.eps = norm->eps;
    a.scale = norm->scale;
    a.T = T;
    a.width = n;
    a.post = block && (norm->flags & SLORA_NORM_POST);
    a.layer = (norm->flags & SLORA_NORM_LAYER) != 0;
    DeviceScope dev(norm->device);
    if (dev.status() != SLORA_OK) return dev.status();
    return launch_norm(a, norm->dtype, (norm->flags & SLORA_NORM_H32) != 0, stream);
}

int32_t slora_w8_quantize(int32_t T, int32_t width, int32_t dtype, int32_t act, const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
                          void *y, int64_t y_stride, int8_t *codes, int64_t codes_stride, float *scales, void *stream)
{
    clear_error();
    if (T < 0) return fail(SLORA_EINVAL, "T=%d is negative", T);
    if (width < 1 || width > SLORA_W8_MAX_WIDTH) return fail(SLORA_EINVAL, "width=%d must be in [1, %d]", width, SLORA_W8_MAX_WIDTH);
    if (dtype != SLORA_F16 && dtype != SLORA_BF16) return fail(SLORA_EINVAL, "unknown dtype %d", dtype);
    if (act != SLORA_ACT_NONE && act != SLORA_ACT_SILU && act != SLORA_ACT_GELU) return fail(SLORA_EINVAL, "unknown act %d", act);
    if (T == 0) return SLORA_OK;
    if ((act != SLORA_ACT_NONE) != (gate != nullptr)) return fail(SLORA_EINVAL, "a gate and its function go together");
    int32_t rc = check_rows("x", x, x_stride, width, kPiece);
    if (rc == SLORA_OK && gate) rc = check_rows("gate", gate, gate_stride, width, kPiece);
    if (rc != SLORA_OK) return rc;
    QuantizeArgs a{};
    a.out = {static_cast<uint16_t *>(y), y_stride, codes, codes_stride, scales};
    if ((rc = check_out(a.out, "y", width)) != SLORA_OK) return rc;
    if (!y && !codes) return fail(SLORA_EINVAL, "y or codes is needed");
    if ((y == x && y_stride != x_stride) || (y && y == gate && y_stride != gate_stride)) return fail(SLORA_EINVAL, "y is x or gate with another stride");
    if (codes && (codes == x || codes == gate)) return fail(SLORA_EINVAL, "codes is the buffer of x or gate");
    a.x = static_cast<const uint16_t *>(x);
    a.gate = static_cast<const uint16_t *>(gate);
    a.x_stride = x_stride;
    a.gate_stride = gate_stride;
    a.T = T;
    a.width = width;
    a.act = act;
    return launch_quantize(a, dtype, stream);
}

} // extern "C"
