// A block's exponent, its codes and their values, in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_device.h"

namespace rc {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float finite_or_zero(float x) { return __builtin_isfinite(x) ? fabsf(x) : 0.f; }

// Largest finite magnitude of 8 bf16 values.
__device__ __forceinline__ float finite_amax8(u32x4 g) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = fmaxf(m, finite_or_zero(bf16_bits_to_float(g[i] & 0xffffu)));
    m = fmaxf(m, finite_or_zero(bf16_bits_to_float(g[i] >> 16)));
  }
  return m;
}

template <int CTRL>
__device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true)));
}

// Maximum over aligned groups of 16 lanes, in every lane.
__device__ __forceinline__ float group_max16(float x) {
  x = dpp_max<0xB1>(x);   // quad_perm [1, 0, 3, 2]
  x = dpp_max<0x4E>(x);   // quad_perm [2, 3, 0, 1]
  x = dpp_max<0x141>(x);  // row_half_mirror
  return dpp_max<0x140>(x);  // row_mirror
}

// e + 127 for the smallest e >= -127 with amax 2^-e <= 448 = 1.75 2^8: amax =
// 1.f 2^(field - 127), so e = field - 135, or one more where 1.f > 1.75.
__device__ __forceinline__ uint32_t exponent_byte(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = int(b >> 23) - 8 + int((b & 0x7fffffu) > 0x600000u);
  return b == 0 ? 127u : uint32_t(max(e, 0));
}

// x 2^-e for the code; what is not finite becomes NaN (the byte is at most 247, so 2^-e is normal).
__device__ __forceinline__ float scaled8(uint32_t bits16, float down) {
  const float x = bf16_bits_to_float(bits16);
  return __builtin_isfinite(x) ? x * down : __builtin_nanf("");
}

__device__ __forceinline__ u32x2 codes8(u32x4 g, uint32_t byte) {
  const float down = __uint_as_float((254u - byte) << 23);
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled8(g[2 * i] & 0xffffu, down), scaled8(g[2 * i] >> 16, down), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled8(g[2 * i + 1] & 0xffffu, down), scaled8(g[2 * i + 1] >> 16, down), w, true);
    out[i] = uint32_t(w);
  }
  return out;
}

// The scale as the conversions take it: they read its exponent field.
__device__ __forceinline__ float scale8(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ u32x4 scaled_values8(u32x2 c, float s) {
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    out[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, false));
    out[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, true));
  }
  return out;
}

// 8 codes times 2^e in bf16.
__device__ __forceinline__ u32x4 values8(u32x2 c, uint32_t byte) { return scaled_values8(c, scale8(byte)); }

// The same for the low byte of any bits: zeros stay zeros whatever lies in place
// of their exponent, 255 (a scale of no number, which no block has) included.
__device__ __forceinline__ u32x4 values8_any(u32x2 c, uint32_t bits) {
  return scaled_values8(c, __uint_as_float(min(bits << 23 & 0x7f800000u, 0x7f000000u)));
}

}  // namespace rc
