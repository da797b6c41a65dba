// The 4-bit cache's format on the device: e2m1 elements, one scale byte (exponent
// + 127) for 32 of them along head_dim.
#pragma once

#include "gfx950_ops.h"

namespace fastvr {
namespace dev {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// What a scale byte multiplies by, as the converting instructions take it: they use
// the exponent field only, with 0 as 2^-127 and 255 as NaN.
static __device__ __forceinline__ float kv4_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// The two values of byte SEL of `codes`, exact in bf16.
template <int SEL>
static __device__ __forceinline__ uint32_t kv4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

// Eight values (four bf16 pairs) of a dword of codes.
static __device__ __forceinline__ u32x4 kv4_values(uint32_t codes, float scale) {
  return u32x4{kv4_pair<0>(codes, scale), kv4_pair<1>(codes, scale), kv4_pair<2>(codes, scale),
               kv4_pair<3>(codes, scale)};
}

}  // namespace dev
}  // namespace fastvr
