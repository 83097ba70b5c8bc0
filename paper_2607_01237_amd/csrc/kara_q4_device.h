// Device side of the 4-bit cache's format (include/kara_q4.h): blocks of 32
// e2m1 codes with one power-of-two scale, which gfx950 converts in hardware.
#pragma once

#include "kara_internal.h"

namespace kara {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kQ4Block = 32;

// 2^(byte - 127), the factor that scale byte 1..254 stands for
__device__ __forceinline__ float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scale byte of a block whose largest magnitude has the fp32 bits `top`
// (finite): adding 0x1fffff carries into the exponent past a mantissa of 1.75,
// that is past 7 units of the scale two binades below.
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t top) {
  const int e = (int)((top + 0x1fffffu) >> 23) - 129;
  return (uint32_t)(min(max(e, -125), 125) + 127);
}

// The pair of values in byte B of `codes`, as two bf16 (exact)
template <int B>
__device__ __forceinline__ uint32_t q4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// The eight values of `codes`, in order
__device__ __forceinline__ bf16x8 q4_octet(uint32_t codes, float scale) {
  const uint4 v = {q4_pair<0>(codes, scale), q4_pair<1>(codes, scale), q4_pair<2>(codes, scale),
                   q4_pair<3>(codes, scale)};
  return __builtin_bit_cast(bf16x8, v);
}

// x as the sum of NT bf16 values: each but the last the upper half of what the ones
// before leave (8 bits of it), the last rounded -- 8, 16 or 24 bits of x.  As fp32
// whose upper halves are the terms.
//
// INF (queries and keys; weights are finite or NaN): an infinity is the last term
// alone.  As the first it would leave inf - inf to the others, and it would meet the
// other factor's lower terms, zeros where one bf16 holds that; the last term meets
// only its first.
template <bool INF, int NT>
__device__ __forceinline__ void bf16_parts(float x, uint32_t (&t)[NT]) {
  uint32_t upper = 0xffff0000u;
  if constexpr (INF && NT > 1) upper = __builtin_isinf(x) ? 0u : upper;
#pragma unroll
  for (int i = 0; i + 1 < NT; ++i) {
    t[i] = __float_as_uint(x) & upper;
    x -= __uint_as_float(t[i]);
  }
  t[NT - 1] = __float_as_uint(x);
}

// Two values' terms as packed pairs, the first value in the lower halves
template <bool INF, int NT>
__device__ __forceinline__ void bf16_term_pairs(float x0, float x1, uint32_t (&t)[NT]) {
  uint32_t a[NT], b[NT];
  bf16_parts<INF>(x0, a);
  bf16_parts<INF>(x1, b);
#pragma unroll
  for (int i = 0; i + 1 < NT; ++i) t[i] = __builtin_amdgcn_perm(b[i], a[i], 0x07060302u);
  const bf16x2 last = {(__bf16)__uint_as_float(a[NT - 1]), (__bf16)__uint_as_float(b[NT - 1])};
  t[NT - 1] = __builtin_bit_cast(uint32_t, last);
}

}  // namespace
}  // namespace kara
