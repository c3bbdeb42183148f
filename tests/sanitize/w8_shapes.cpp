// Which shape of tiles a product takes, and whether its weights are loaded without a place in the caches: matrices, outputs, inputs and tokens of each call come as
// arguments, the answers go out a line each.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>

#include "w8.hpp"

extern "C" {
hipError_t hipGetDevice(int *) { return hipErrorNoDevice; }
const char *hipGetErrorString(hipError_t) { return "stand-in"; }
}
namespace slora {
int32_t fail(int32_t code, const char *, ...) { return code; }
void clear_error() {}
DeviceScope::DeviceScope(int) {}
DeviceScope::~DeviceScope() {}
int32_t launch_w8_pack(const slora_w8 *, const int8_t *, const float *, void *, void *) { return SLORA_OK; }
int32_t launch_w8(W8Args &, int, void *) { return SLORA_OK; }
} // namespace slora

int main(int argc, char **argv)
{
    for (int i = 1; i + 3 < argc; i += 4) {
        slora::W8Args a{};
        a.n = std::atoi(argv[i]);
        for (int k = 0; k < a.n; ++k) {
            a.m[k].outputs = std::atoi(argv[i + 1]);
            a.m[k].tiles = (a.m[k].outputs + kW8Rows - 1) / kW8Rows;
            a.m[k].chunks = (std::atoi(argv[i + 2]) + 2 * kW8Chunk - 1) / (2 * kW8Chunk) * 2;
        }
        a.T = std::atoi(argv[i + 3]);
        const slora::W8Shape &s = slora::kW8Shapes[slora::w8_shape(a)];
        std::printf("%d %d %d\n", s.outputs, s.tokens, (int)slora::w8_once(a, s));
    }
    std::printf("%d shapes\n", (int)(sizeof(slora::kW8Shapes) / sizeof(slora::kW8Shapes[0])));
    return 0;
}
