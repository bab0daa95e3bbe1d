// A block's exponent, its codes and their values, in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_device.h"

namespace rc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// Magnitudes of bf16 order like their bits without the sign; 0x7f80 and above is not finite.
__device__ __forceinline__ uint32_t abs_max8(u32x4 g) {
  u16x2 m{0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, g[i] & 0x7fff7fffu));
  return max(uint32_t(m[0]), uint32_t(m[1]));
}

__device__ __forceinline__ uint32_t finite_abs_max8(u32x4 g) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = g[i] & 0x7fffu, hi = g[i] >> 16 & 0x7fffu;
    m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  return m;
}

// Largest finite magnitude of each of N granules, as bits.  Values that are not
// finite are rare: a wave looks for them one by one only where it has met some.
template <int N>
__device__ __forceinline__ void finite_abs_max(const u32x4 (&g)[N], uint32_t (&m)[N]) {
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) all = max(all, m[i] = abs_max8(g[i]));
  if (__any(all >= 0x7f80u)) {
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = finite_abs_max8(g[i]);
  }
}

// The largest of them all.
template <int N>
__device__ __forceinline__ uint32_t finite_abs_max(const u32x4 (&g)[N]) {
  uint32_t m[N], all = 0;
  finite_abs_max(g, m);
#pragma unroll
  for (int i = 0; i < N; ++i) all = max(all, m[i]);
  return all;
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  return max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xf, 0xf, true)));
}

// Maximum over aligned groups of 16 lanes, in every lane.
__device__ __forceinline__ uint32_t group_max16(uint32_t x) {
  x = dpp_max<0xB1>(x);   // quad_perm [1, 0, 3, 2]
  x = dpp_max<0x4E>(x);   // quad_perm [2, 3, 0, 1]
  x = dpp_max<0x141>(x);  // row_half_mirror
  return dpp_max<0x140>(x);  // row_mirror
}

// e + 127 for the smallest e >= -127 with amax 2^-e <= 448 = 1.75 2^8, of the bits of
// amax = 1.f 2^(field - 127): e = field - 135, or one more where 1.f > 1.75 (f > 0x60 / 0x80).
__device__ __forceinline__ uint32_t exponent_byte(uint32_t amax) {
  return amax == 0 ? 127u : uint32_t(max(int((amax + 0x1fu) >> 7) - 8, 0));
}

// The scale as the conversions take it: they read its exponent field.
__device__ __forceinline__ float scale8(uint32_t byte) { return __uint_as_float(byte << 23); }

// Of the low byte of any bits: finite whatever lies in place of the exponent, 255 (a
// scale of no number, which no block has) included, so that zeros stay zeros.
__device__ __forceinline__ float scale8_any(uint32_t bits) {
  return __uint_as_float(min(bits << 23 & 0x7f800000u, 0x7f000000u));
}

// The low or high two of four codes times the scale, in bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t widened(uint32_t codes, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s, HIGH));
}

// Codes of 8 bf16 values: the conversion takes 2^e out exactly, rounds to nearest
// (ties to even), and makes NaN of what is not finite.
__device__ __forceinline__ u32x2 codes8(u32x4 g, uint32_t byte) {
  const float s = scale8(byte);
  const bf16x8 v = __builtin_bit_cast(bf16x8, g);
  i16x2 lo{0, 0}, hi{0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_shufflevector(v, v, 0, 1), s, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_shufflevector(v, v, 2, 3), s, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_shufflevector(v, v, 4, 5), s, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_shufflevector(v, v, 6, 7), s, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// 8 codes times 2^e in bf16.
__device__ __forceinline__ u32x4 values8(u32x2 c, uint32_t byte) {
  const float s = scale8(byte);
  return u32x4{widened<false>(c[0], s), widened<true>(c[0], s), widened<false>(c[1], s), widened<true>(c[1], s)};
}

}  // namespace rc
