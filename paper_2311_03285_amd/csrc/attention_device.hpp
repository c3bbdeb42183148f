// What the kernels of the 8-bit KV cache, of the 4-bit and 8-bit products and of whole rows share.
#pragma once

#include <hip/hip_runtime.h>

#include "slora_internal.hpp"

namespace slora {

namespace {

constexpr int kWave = 64;

template <int DT>
__device__ __forceinline__ float widen(uint16_t b)
{
    return DT == SLORA_F16 ? (float)__builtin_bit_cast(_Float16, b) : __uint_as_float((uint32_t)b << 16);
}
template <int DT>
__device__ __forceinline__ uint16_t narrow(float f)
{
    if constexpr (DT == SLORA_F16)
        return __builtin_bit_cast(uint16_t, (_Float16)f);
    else
        return __builtin_bit_cast(uint16_t, (__bf16)f);
}

// the wavefront's number in its workgroup, as a scalar: what follows from it takes no vector instructions
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave); }

int32_t check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SLORA_OK : fail(SLORA_EHIP, "launching %s: %s", what, hipGetErrorString(e));
}

} // namespace

} // namespace slora
