// Which shape of tiles a product takes: outputs and tokens of each call come in pairs as arguments, the shapes go out a line each.
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
    for (int i = 1; i + 1 < argc; i += 2) {
        slora::W8Args a{};
        a.n = 1;
        a.m[0].outputs = std::atoi(argv[i]);
        a.T = std::atoi(argv[i + 1]);
        const slora::W8Shape &s = slora::kW8Shapes[slora::w8_shape(a)];
        std::printf("%d %d\n", s.outputs, s.tokens);
    }
    std::printf("%d shapes\n", (int)(sizeof(slora::kW8Shapes) / sizeof(slora::kW8Shapes[0])));
    return 0;
}
