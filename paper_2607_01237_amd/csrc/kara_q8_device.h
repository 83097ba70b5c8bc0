// Device side of the 8-bit cache's format (include/kara_q8.h): e4m3 codes under one
// power-of-two scale for a page's rows of a KV head, which gfx950 converts in hardware.
#pragma once

#include "kara_q4_device.h"

namespace kara {
namespace {

constexpr uint32_t kQ8Lowest = 10;    // scale byte of a block of zeros: 2^-117
constexpr uint32_t kQ8Highest = 246;  // 2^119

// Scale byte of a block whose largest magnitude has the fp32 bits `top` (finite): adding
// 0x1fffff carries into the exponent past a mantissa of 1.75, that is past 448 units of
// the scale eight binades below.
__device__ __forceinline__ uint32_t q8_scale_byte(uint32_t top) {
  const int b = (int)((top + 0x1fffffu) >> 23) - 8;
  return (uint32_t)min(max(b, (int)kQ8Lowest), (int)kQ8Highest);
}

// 2^(byte - 127) and its inverse.  (A page that nothing was written to may hold any byte:
// what is read with it is not used, and no shift leaves 32 bits.)
__device__ __forceinline__ float q8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float q8_per_unit(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Two codes of `codes` (its lower or upper half) as two bf16, exact
template <bool HI>
__device__ __forceinline__ uint32_t q8_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}

// Eight codes, in order
__device__ __forceinline__ bf16x8 q8_octet(uint32_t lo, uint32_t hi, float scale) {
  const uint4 v = {q8_pair<false>(lo, scale), q8_pair<true>(lo, scale), q8_pair<false>(hi, scale),
                   q8_pair<true>(hi, scale)};
  return __builtin_bit_cast(bf16x8, v);
}

// Four finite or infinite values to codes; per_unit: q8_per_unit of the scale
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, float per_unit) {
  auto units = [&](float x) { return __builtin_amdgcn_fmed3f(x * per_unit, -448.f, 448.f); };
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(units(a), units(b), w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(units(c), units(d), w, true);
  return (uint32_t)w;
}

// Four codes under one scale to codes under a larger one
__device__ __forceinline__ uint32_t q8_rescale(uint32_t codes, float ratio) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return q8_codes(lo[0], lo[1], hi[0], hi[1], ratio);
}

}  // namespace
}  // namespace kara
