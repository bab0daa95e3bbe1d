// Sums across lanes without LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rc {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// Sum over aligned groups of L = 8 or 16 lanes, in every lane: neighbours, pairs
// of a quad, quads (mirrored halves of 8), halves of 16.
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  static_assert(L == 8 || L == 16, "groups of a DPP row");
  x = dpp_add<0xB1>(x);   // quad_perm [1, 0, 3, 2]
  x = dpp_add<0x4E>(x);   // quad_perm [2, 3, 0, 1]
  x = dpp_add<0x141>(x);  // row_half_mirror
  if (L == 16) x = dpp_add<0x140>(x);  // row_mirror
  return x;
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
  x = group_sum<16>(x);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace rc
