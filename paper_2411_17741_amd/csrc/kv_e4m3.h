// Pages of 8-bit values on the device (gfx950): e4m3 values and the power of two that those of a token and head are multiplied by.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace lora {

struct E4m3 {
    uint8_t bits;
};

// what an exponent byte says (1 to 254)
__device__ __forceinline__ float unit_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }
__device__ __forceinline__ float value_of(E4m3 v) { return __builtin_amdgcn_cvt_f32_fp8(v.bits, 0); }

// 8 values of 8 bits times a unit as bf16
__device__ __forceinline__ uint4 eight_bf16(uint32_t a, uint32_t b, float unit)
{
    const auto two = [&](uint32_t v, auto high) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, unit, decltype(high)::value)); };
    return make_uint4(two(a, std::false_type{}), two(a, std::true_type{}), two(b, std::false_type{}), two(b, std::true_type{}));
}

}  // namespace lora
