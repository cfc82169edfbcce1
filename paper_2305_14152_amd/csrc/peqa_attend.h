// What the attention kernels have in common: matrix instructions on operands as they are in registers, lane exchanges, 8-bit floats.
#pragma once

#include "peqa_device.h"

namespace peqa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float LOWEST = -3.0e38f;       // finite stand-in for the maximum of nothing: e^(-inf - LOWEST) is 0, not NaN
constexpr float LN2 = 0.693147180559945309f, LOG2E = 1.44269504088896341f;

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 x, u32x4 y, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(u32x4 x, u32x4 y, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// f over the four lanes of a wave with the same lane % 16, in all of them: rows of 16 lanes change places, then halves.
template <typename F> __device__ __forceinline__ float across_groups(float v, F f)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Four 8-bit floats as bf16, or two as fp16: exact.
template <bool HI> __device__ __forceinline__ uint32_t fp8_bf16(uint32_t v)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, HI));
}
template <bool HI> __device__ __forceinline__ uint32_t fp8_f16(uint32_t v)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, HI));
}

}  // namespace peqa
