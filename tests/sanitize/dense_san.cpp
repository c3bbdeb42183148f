// Host code of the norms, of rows in 8 bits and of the products with 8-bit weights under AddressSanitizer / UndefinedBehaviorSanitizer, on the CPU only.
//
// rows.cpp and w8.cpp are compiled unchanged; the stand-in launchers check what the kernels assume of their arguments.  Every refusal is made
// once, with the rest of the call as it should be: nothing may be launched.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>

#include "rows.hpp"
#include "w8.hpp"

#define REQUIRE(c)                                                                   \
    do {                                                                             \
        if (!(c)) {                                                                  \
            std::fprintf(stderr, "dense_san: %s failed at line %d\n", #c, __LINE__); \
            std::abort();                                                            \
        }                                                                            \
    } while (0)

static bool g_no_device = false;
static long g_launches = 0;
static char g_text[512];

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return g_no_device ? hipErrorNoDevice : hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stand-in"; }
}

namespace slora {
int32_t fail(int32_t code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_text, sizeof g_text, fmt, ap);
    va_end(ap);
    return code;
}
void clear_error() { g_text[0] = 0; }
const char *last_error_cstr() { return g_text; }
DeviceScope::DeviceScope(int device) { REQUIRE(device == 0); }
DeviceScope::~DeviceScope() {}

static void check_out(const RowsOut &o, int32_t width)
{
    if (o.x) REQUIRE(((uintptr_t)o.x & 15) == 0 && o.x_stride >= width && o.x_stride % 8 == 0);
    if (o.codes) REQUIRE(((uintptr_t)o.codes & 15) == 0 && o.codes_stride >= width && o.codes_stride % 16 == 0 && o.scales);
}
int32_t launch_norm(const NormArgs &a, int32_t dtype, bool, void *)
{
    ++g_launches;
    REQUIRE(a.T > 0 && a.width >= 1 && a.width <= SLORA_NORM_MAX_WIDTH && (dtype == SLORA_F16 || dtype == SLORA_BF16));
    REQUIRE(a.h && a.h_stride >= a.width && a.h_stride % 8 == 0 && ((uintptr_t)a.h & 15) == 0);
    if (a.block) REQUIRE(a.block_stride >= a.width && a.block_stride % 8 == 0);
    if (a.gate) REQUIRE(a.block && (a.gate_stride == 0 || (a.gate_stride >= a.width && a.gate_stride % 8 == 0)));
    REQUIRE(!a.post || a.block);
    REQUIRE(a.h_out || a.out.x || a.out.codes);
    check_out(a.out, a.width);
    return SLORA_OK;
}
int32_t launch_quantize(const QuantizeArgs &a, int32_t, void *)
{
    ++g_launches;
    REQUIRE(a.T > 0 && a.width >= 1 && a.width <= SLORA_W8_MAX_WIDTH && a.x && (a.gate != nullptr) == (a.act != SLORA_ACT_NONE));
    REQUIRE(a.out.x || a.out.codes);
    check_out(a.out, a.width);
    return SLORA_OK;
}
int32_t launch_w8_pack(const slora_w8 *w, const int8_t *, const float *, void *, void *)
{
    ++g_launches;
    REQUIRE(w->chunks % 2 == 0 && (int64_t)w->chunks * kW8Chunk >= w->inputs && (int64_t)w->tiles * kW8Rows >= w->outputs);
    return SLORA_OK;
}
int32_t launch_w8(W8Args &a, int y, void *)
{
    ++g_launches;
    REQUIRE(a.n >= 1 && a.n <= SLORA_MAX_MULTI && a.T > 0 && a.T <= 1 << 30 && y >= 0 && y <= 2);
    for (int32_t k = 0; k < a.n; ++k) {
        const W8Matrix &m = a.m[k];
        REQUIRE(m.codes && m.x && m.scales && m.x_scales && m.y && m.x_last % 16 == 0 && m.x_last + 16 <= m.x_stride && m.x_stride <= kW8MostStride);
        // rows of a workgroup, and offsets behind its stages, stay below the offset that loads nothing
        REQUIRE((int64_t)255 * m.x_stride + m.x_last + 16 + 8 * 128 < (int64_t)1 << 30 && (int64_t)16 * m.chunks * kW8Block + 8 * 2048 < (int64_t)1 << 30);
        REQUIRE(m.y_stride >= m.outputs);
    }
    return SLORA_OK;
}
} // namespace slora

static char *const P = reinterpret_cast<char *>(0x10000); // addresses that nobody reads
static void *at(int64_t n) { return P + n; }
static uint16_t *v16(int64_t n) { return reinterpret_cast<uint16_t *>(P + n); }

struct Refused {
    long before = g_launches;
    void operator()(int32_t rc, int32_t want) const
    {
        REQUIRE(rc == want);
        REQUIRE(g_text[0] != 0 && g_launches == before);
    }
};

static void norms()
{
    const float nan = std::numeric_limits<float>::quiet_NaN(), inf = std::numeric_limits<float>::infinity();
    slora_norm *n = nullptr;
    const Refused no;
    no(slora_norm_init(nullptr, 64, 0, 0, 1e-5f, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    for (int width : {0, -1, SLORA_NORM_MAX_WIDTH + 1}) no(slora_norm_init(&n, width, 0, 0, 1e-5f, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    no(slora_norm_init(&n, 64, 2, 0, 1e-5f, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    for (int flags : {8, -1}) no(slora_norm_init(&n, 64, 0, flags, 1e-5f, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    for (float eps : {-1.0f, nan, inf, 1e-20f}) no(slora_norm_init(&n, 64, 0, 0, eps, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    for (float scale : {nan, inf}) no(slora_norm_init(&n, 64, 0, 0, 0, scale, nullptr, nullptr, nullptr, nullptr), SLORA_EINVAL);
    no(slora_norm_init(&n, 64, 0, 0, 0, 1, at(16), nullptr, nullptr, nullptr), SLORA_EINVAL);
    no(slora_norm_init(&n, 64, 0, 0, 0, 1, nullptr, at(16), nullptr, nullptr), SLORA_EINVAL);
    no(slora_norm_init(&n, 64, 0, 0, 0, 1, nullptr, nullptr, at(2), nullptr), SLORA_EINVAL);
    no(slora_norm_init(&n, 64, 0, 0, 0, 1, nullptr, nullptr, nullptr, at(8)), SLORA_EINVAL);
    g_no_device = true;
    no(slora_norm_init(&n, 64, 0, 0, 0, 1, nullptr, nullptr, nullptr, nullptr), SLORA_EHIP);
    g_no_device = false;
    REQUIRE(n == nullptr && slora_norm_destroy(nullptr) == SLORA_OK);

    REQUIRE(slora_norm_init(&n, 60, SLORA_BF16, SLORA_NORM_POST, 1e-5f, 0.5f, at(16), at(32), at(48), at(64)) == SLORA_OK);
    struct Call {
        int32_t T = 3;
        void *h = at(0x1000);
        int64_t h_stride = 64;
        void *block = at(0x2000);
        int64_t block_stride = 64;
        void *gate = at(0x3000);
        int64_t gate_stride = 0;
        void *h_out = at(0x4000);
        int64_t h_out_stride = 64;
        void *x = at(0x5000);
        int64_t x_stride = 64;
        int8_t *codes = reinterpret_cast<int8_t *>(at(0x6000));
        int64_t codes_stride = 64;
        float *scales = reinterpret_cast<float *>(at(0x7000));
        int32_t operator()(slora_norm *n) const
        {
            return slora_norm_apply(n, T, h, h_stride, block, block_stride, gate, gate_stride, h_out, h_out_stride, x, x_stride, codes, codes_stride, scales, nullptr);
        }
    };
    long launched = g_launches;
    auto ok = [&](auto change) {
        Call c;
        change(c);
        REQUIRE(c(n) == SLORA_OK && g_launches == ++launched);
    };
    ok([](Call &) {});
    ok([](Call &c) { c.gate = nullptr; });
    ok([](Call &c) { c.gate_stride = 72; });
    ok([](Call &c) { c.block = c.gate = nullptr; });
    ok([](Call &c) { c.h_out = c.h; });
    ok([](Call &c) { c.x = c.block; });
    ok([](Call &c) { c.h_out = nullptr; c.x = nullptr; });
    ok([](Call &c) { c.codes = nullptr; c.scales = nullptr; });
    {
        Call c;
        c.T = 0;
        c.h = nullptr;
        REQUIRE(c(n) == SLORA_OK && g_launches == launched); // no tokens, no work
    }
    auto bad = [&](auto change) {
        Call c;
        change(c);
        const Refused refused;
        refused(c(n), SLORA_EINVAL);
    };
    {
        const Refused refused;
        refused(Call()(nullptr), SLORA_EINVAL);
    }
    bad([](Call &c) { c.T = -1; });
    bad([](Call &c) { c.h = nullptr; });
    bad([](Call &c) { c.gate_stride = 16; });
    bad([](Call &c) { c.gate_stride = -64; });
    bad([](Call &c) { c.block = nullptr; }); // a gate without a block
    bad([](Call &c) { c.h_out = c.h; c.h_out_stride = 72; });
    bad([](Call &c) { c.x = c.block; c.x_stride = 72; });
    bad([](Call &c) { c.x = c.h; });
    bad([](Call &c) { c.x = c.h_out; });
    bad([](Call &c) { c.h_out = c.block; });
    bad([](Call &c) { c.codes = (int8_t *)c.x; });
    bad([](Call &c) { c.codes = (int8_t *)c.h_out; });
    bad([](Call &c) { c.scales = nullptr; });
    bad([](Call &c) { c.codes = nullptr; });
    bad([](Call &c) { c.scales = (float *)at(0x7002); });
    bad([](Call &c) { c.h_out = c.x = nullptr; c.codes = nullptr; c.scales = nullptr; });
    for (int64_t stride : {(int64_t)56, (int64_t)60, (int64_t)0, (int64_t)-64, (int64_t)1 << 30, std::numeric_limits<int64_t>::min()}) {
        bad([=](Call &c) { c.h_stride = stride; });
        bad([=](Call &c) { c.block_stride = stride; });
        bad([=](Call &c) { c.h_out_stride = stride; });
        bad([=](Call &c) { c.x_stride = stride; });
        bad([=](Call &c) { c.codes_stride = stride; });
    }
    bad([](Call &c) { c.codes_stride = 72; });
    bad([](Call &c) { c.h = at(0x1008); });
    bad([](Call &c) { c.block = at(0x2008); });
    bad([](Call &c) { c.gate = at(0x3002); });
    bad([](Call &c) { c.h_out = at(0x4008); });
    bad([](Call &c) { c.x = at(0x5008); });
    bad([](Call &c) { c.codes = (int8_t *)at(0x6008); });
    REQUIRE(slora_norm_destroy(n) == SLORA_OK);
}

static void rows()
{
    struct Call {
        int32_t T = 2, width = 100, dtype = SLORA_F16, act = SLORA_ACT_SILU;
        void *x = at(0x1000);
        int64_t x_stride = 104;
        void *gate = at(0x2000);
        int64_t gate_stride = 104;
        void *y = at(0x3000);
        int64_t y_stride = 104;
        int8_t *codes = reinterpret_cast<int8_t *>(at(0x4000));
        int64_t codes_stride = 112;
        float *scales = reinterpret_cast<float *>(at(0x5000));
        int32_t operator()() const { return slora_w8_quantize(T, width, dtype, act, x, x_stride, gate, gate_stride, y, y_stride, codes, codes_stride, scales, nullptr); }
    };
    long launched = g_launches;
    auto ok = [&](auto change) {
        Call c;
        change(c);
        REQUIRE(c() == SLORA_OK && g_launches == ++launched);
    };
    auto bad = [&](auto change) {
        Call c;
        change(c);
        const Refused refused;
        refused(c(), SLORA_EINVAL);
    };
    ok([](Call &) {});
    ok([](Call &c) { c.y = c.x; });
    ok([](Call &c) { c.y = c.gate; });
    ok([](Call &c) { c.y = nullptr; });
    ok([](Call &c) { c.codes = nullptr; c.scales = nullptr; });
    ok([](Call &c) { c.act = SLORA_ACT_NONE; c.gate = nullptr; });
    ok([](Call &c) { c.width = SLORA_W8_MAX_WIDTH; c.x_stride = c.gate_stride = c.y_stride = c.codes_stride = SLORA_W8_MAX_WIDTH; });
    {
        Call c;
        c.T = 0;
        c.x = nullptr;
        REQUIRE(c() == SLORA_OK && g_launches == launched);
    }
    bad([](Call &c) { c.T = -1; });
    for (int width : {0, -1, SLORA_W8_MAX_WIDTH + 1}) bad([=](Call &c) { c.width = width; });
    bad([](Call &c) { c.dtype = 2; });
    for (int act : {3, -1}) bad([=](Call &c) { c.act = act; });
    bad([](Call &c) { c.act = SLORA_ACT_NONE; });
    bad([](Call &c) { c.gate = nullptr; });
    bad([](Call &c) { c.x = nullptr; });
    bad([](Call &c) { c.y = nullptr; c.codes = nullptr; c.scales = nullptr; });
    bad([](Call &c) { c.scales = nullptr; });
    bad([](Call &c) { c.y = c.x; c.y_stride = 112; });
    bad([](Call &c) { c.y = c.gate; c.y_stride = 112; });
    bad([](Call &c) { c.codes = (int8_t *)c.x; });
    bad([](Call &c) { c.codes = (int8_t *)c.gate; });
    bad([](Call &c) { c.codes = (int8_t *)c.y; });
    for (int64_t stride : {(int64_t)96, (int64_t)102, (int64_t)-104}) {
        bad([=](Call &c) { c.x_stride = stride; });
        bad([=](Call &c) { c.gate_stride = stride; });
        bad([=](Call &c) { c.y_stride = stride; });
        bad([=](Call &c) { c.codes_stride = stride; });
    }
    bad([](Call &c) { c.codes_stride = 104; });
    bad([](Call &c) { c.x = at(0x1004); });
    bad([](Call &c) { c.gate = at(0x2004); });
    bad([](Call &c) { c.y = at(0x3004); });
}

static void products()
{
    int64_t bytes = 0;
    const Refused no;
    no(slora_w8_bytes(4, 4, nullptr), SLORA_EINVAL);
    for (int outputs : {0, -1, (1 << 24) + 1}) no(slora_w8_bytes(outputs, 64, &bytes), SLORA_EINVAL);
    for (int inputs : {0, -5, SLORA_W8_MAX_INPUTS + 1}) no(slora_w8_bytes(16, inputs, &bytes), SLORA_EINVAL);
    REQUIRE(slora_w8_bytes(17, 129, &bytes) == SLORA_OK && bytes == 2 * 4 * 1024 + 32 * 4);
    REQUIRE(slora_w8_bytes(1 << 24, SLORA_W8_MAX_INPUTS, &bytes) == SLORA_OK && bytes == ((int64_t)1 << 20) * 2048 * 1024 + ((int64_t)4 << 24));
    slora_w8 *w = nullptr, *other = nullptr;
    const int8_t *codes = reinterpret_cast<int8_t *>(at(0x101)); // any address
    const float *scales = reinterpret_cast<float *>(at(0x200));
    no(slora_w8_pack(nullptr, 40, 100, 0, codes, scales, at(0x1000), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 5, codes, scales, at(0x1000), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 0, 0, codes, scales, at(0x1000), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 0, nullptr, scales, at(0x1000), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 0, codes, nullptr, at(0x1000), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 0, codes, scales, nullptr, nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 0, codes, scales, at(0x1008), nullptr), SLORA_EINVAL);
    no(slora_w8_pack(&w, 40, 100, 0, codes, reinterpret_cast<float *>(at(0x201)), at(0x1000), nullptr), SLORA_EINVAL);
    g_no_device = true;
    no(slora_w8_pack(&w, 40, 100, 0, codes, scales, at(0x1000), nullptr), SLORA_EHIP);
    g_no_device = false;
    REQUIRE(w == nullptr && slora_w8_destroy(nullptr) == SLORA_OK);
    REQUIRE(slora_w8_pack(&w, 40, 100, SLORA_F16, codes, scales, at(0x1000), nullptr) == SLORA_OK);
    REQUIRE(slora_w8_pack(&other, 40, SLORA_W8_MAX_INPUTS, SLORA_BF16, codes, scales, at(0x9000), nullptr) == SLORA_OK);

    struct Call {
        int32_t n = 2, T = 5;
        const slora_w8 *w[9];
        const int8_t *x[9];
        int64_t x_stride[9], y_stride[9];
        const float *x_scales[9];
        void *y[9];
        bool missing = false;
        int32_t operator()(bool y16) const
        {
            const int64_t *xs = missing ? nullptr : x_stride;
            return y16 ? slora_w8_matmul_y16(n, w, x, xs, x_scales, T, y, y_stride, nullptr)
                       : slora_w8_matmul(n, w, x, xs, x_scales, T, reinterpret_cast<float *const *>(y), y_stride, nullptr);
        }
    };
    Call good;
    for (int k = 0; k < 9; ++k) {
        good.w[k] = w;
        good.x[k] = reinterpret_cast<int8_t *>(at(0x10000));
        good.x_stride[k] = 112;
        good.x_scales[k] = reinterpret_cast<float *>(at(0x20000));
        good.y[k] = at(0x30000 + 0x1000 * k);
        good.y_stride[k] = 40 + k;
    }
    long launched = g_launches;
    auto ok = [&](auto change) {
        for (bool y16 : {false, true}) {
            Call c = good;
            change(c);
            REQUIRE(c(y16) == SLORA_OK && g_launches == ++launched);
        }
    };
    auto bad = [&](auto change, int32_t code = SLORA_EINVAL) {
        for (bool y16 : {false, true}) {
            Call c = good;
            change(c);
            const Refused refused;
            refused(c(y16), code);
        }
    };
    ok([](Call &) {});
    ok([](Call &c) { c.n = 8; });
    ok([](Call &c) { c.x_stride[1] = slora::kW8MostStride; });
    ok([&](Call &c) { c.n = 1; c.w[0] = other; c.x_stride[0] = 131072; });
    ok([](Call &c) { c.T = 1 << 30; });
    {
        Call c = good;
        c.T = 0;
        c.x[0] = nullptr;
        REQUIRE(c(true) == SLORA_OK && g_launches == launched);
    }
    for (int n : {0, -1, 9}) bad([=](Call &c) { c.n = n; });
    bad([](Call &c) { c.T = -1; });
    bad([](Call &c) { c.T = (1 << 30) + 1; }, SLORA_ERANGE);
    bad([](Call &c) { c.missing = true; });
    bad([](Call &c) { c.w[1] = nullptr; });
    bad([&](Call &c) { c.w[1] = other; });
    bad([](Call &c) { c.x[1] = nullptr; });
    bad([](Call &c) { c.x_scales[1] = nullptr; });
    bad([](Call &c) { c.y[1] = nullptr; });
    bad([](Call &c) { c.y[1] = c.y[0]; });
    bad([](Call &c) { c.x[1] += 8; });
    bad([](Call &c) { c.y[1] = at(0x30008); });
    bad([](Call &c) { c.x_scales[0] = reinterpret_cast<float *>(at(0x20002)); });
    for (int64_t stride : {(int64_t)96, (int64_t)104, (int64_t)0, (int64_t)-112, slora::kW8MostStride + 16, std::numeric_limits<int64_t>::max()}) bad([=](Call &c) { c.x_stride[1] = stride; });
    for (int64_t stride : {(int64_t)39, (int64_t)0, (int64_t)-40, ((int64_t)1 << 29) + 1}) bad([=](Call &c) { c.y_stride[1] = stride; });
    REQUIRE(slora_w8_destroy(w) == SLORA_OK && slora_w8_destroy(other) == SLORA_OK);
}

int main()
{
    norms();
    rows();
    products();
    std::printf("dense_san OK: %ld launches\n", g_launches);
    return 0;
}
