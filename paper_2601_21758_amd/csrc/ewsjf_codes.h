// e4m3 codes and their scales, on the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ewsjf {

template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));

// 2^(byte - 127) of a scale byte in [1, 254].
__device__ inline float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// Eight codes to values: exact where the type holds them.
__device__ inline vec8<__bf16> values_of(uint2 codes, float scale, __bf16) {
  const uint4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, true))};
  return __builtin_bit_cast(vec8<__bf16>, v);
}
__device__ inline vec8<_Float16> values_of(uint2 codes, float scale, _Float16) {
  const uint4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes.x, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes.x, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes.y, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes.y, scale, true))};
  return __builtin_bit_cast(vec8<_Float16>, v);
}

}  // namespace ewsjf
