// Pages of 8-bit values on the device (gfx950): e4m3 values and the power of two that those of a token and head are multiplied by.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace lora {

struct E4m3 {
    uint8_t bits;
};

// what an exponent byte says (1 to 254)
__device__ __forceinline__ float unit_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }
__device__ __forceinline__ float value_of(E4m3 v) { return __builtin_amdgcn_cvt_f32_fp8(v.bits, 0); }

}  // namespace lora
