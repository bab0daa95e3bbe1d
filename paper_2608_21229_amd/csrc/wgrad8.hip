// Gradient of a projection's weights from an 8-bit checkpoint of its input:
//
//   dw[n, k] = sum_m dy[m, n] x[m, k],  x = code 2^e, dy in bf16, fp32 sums and result
//
// The codes are widened to bf16 (exact) on their way into LDS, so the product is
// one of v_mfma_f32_32x32x16_bf16.  The sum runs over rows, which both operands
// hold as their slow dimension: the fragments are read with the transpose read
// ds_read_b64_tr_b16 (16 lanes take 4 rows of 16 columns, each lane a column).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_blocks8.h"
#include "rc_lds.h"
#include "rc_quant8.h"

namespace rc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr int kSlice = 64;  // rows per step

// Granule g (8 columns) of row r lies at slot g ^ swz(r): the four rows of a
// transpose read fall into four quarters of the banks.
__device__ __forceinline__ int swz(int row) { return (row & 3) << 2 | (row >> 2 & 3); }

// Columns c0 + lane % 32 of 16 rows from r0 on, a tile with C columns per row.
template <int C>
__device__ __forceinline__ bf16x8 tr_frag(const char* t, int r0, int c0, int lane) {
  const int li = lane & 15, row = r0 + 4 * (lane >> 5) + (li >> 2);
  const int g = c0 / 8 + 2 * (lane >> 4 & 1) + ((li & 3) >> 1);
  const char* lo = t + row * C * 2 + 16 * (g ^ swz(row)) + 8 * (li & 1);
  const char* hi = t + (row + 8) * C * 2 + 16 * (g ^ swz(row + 8)) + 8 * (li & 1);
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)lo);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)hi);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One tile of n x k and one share of the rows per work-group: WN x WK waves,
// each NB x KB accumulators of 32 x 32.
template <int NB, int KB, int WN, int WK>
__global__ __launch_bounds__(WN * WK * 64) void wgrad8_kernel(const WGrad8Params q) {
  constexpr int NW = WN * WK;
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK;
  constexpr int kDy = kSlice * TN * 2, kX = kSlice * TK * 2, kStage = kDy + kX;
  constexpr int CD = kDy / 1024 / NW;            // 1 KB chunks of dy per wave
  constexpr int GX = TK / 8;                     // granules of a row of x
  constexpr int RQ = kSlice / 4;                 // groups of four rows
  constexpr int IX = RQ * GX / (NW * 64);        // groups per thread
  static_assert(CD * NW * 1024 == kDy && IX * NW * 64 == RQ * GX && NW * 64 % GX == 0, "loads divide over the waves");
  __shared__ __attribute__((aligned(1024))) char ring[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave / WK, wk = wave % WK;

  const int64_t rows_n = (q.N + TN - 1) / TN, cols_k = (q.K + TK - 1) / TK, tiles = rows_n * cols_k;
  const int64_t w = xcd_block(blockIdx.x, gridDim.x);
  const int split = int(w / tiles);
  int64_t tn, tk;
  grouped_tile(w % tiles, rows_n, cols_k, 4, tn, tk);
  const int n0 = int(tn * TN), k0 = int(tk * TK);
  const int64_t slices = (q.M + kSlice - 1) / kSlice;
  const int64_t s0 = slices * split / q.splits, s1 = slices * (split + 1) / q.splits;

  // dy: lane l of chunk c fills slot 64 c + l
  constexpr int GD = TN / 8;
  uint32_t doff[CD];
#pragma unroll
  for (int i = 0; i < CD; ++i) {
    const int p = (i * NW + wave) * 64 + lane, row = p / GD;
    doff[i] = uint32_t(row) * uint32_t(q.lddy) * 2u + uint32_t((p % GD) ^ swz(row)) * 16u;
  }
  const int64_t dy_cols = min(TN, q.N - n0) * 2;
  const auto issue_dy = [&](int64_t s, uint32_t stage) {
    const int64_t m = s * kSlice, rows = min(int64_t(kSlice), q.M - m);
    const __amdgpu_buffer_rsrc_t r = bytes_rsrc(q.dy + m * q.lddy + n0, (rows - 1) * q.lddy * 2 + dy_cols);
#pragma unroll
    for (int i = 0; i < CD; ++i) dma16(lds_u32(ring) + stage + uint32_t((i * NW + wave) * 1024), doff[i], r);
  };

  // x: a thread takes 8 codes of four consecutive rows, whose exponents are one dword
  const int gx = tid % GX, rq = tid / GX;
  const int kblocks = int(blocks8(q.K)), kb0 = k0 / kBlock8;
  const int dkb = min(gx * 8 / kBlock8, kblocks - 1 - kb0);
  const int64_t x_cols = min(TK, kblocks * kBlock8 - k0);
  u32x2 xc[IX][4];
  uint32_t xe[IX];
  const auto load_x = [&](int64_t s) {
    const int64_t m = s * kSlice, rows = min(int64_t(kSlice), q.M - m);
    const __amdgpu_buffer_rsrc_t r = bytes_rsrc(q.x.codes + m * q.x.ld + k0, (rows - 1) * q.x.ld + x_cols);
    const __amdgpu_buffer_rsrc_t e = bytes_rsrc(q.x.exps + kb0 * q.x.le + m, min(int64_t(0x7fffffff), (kblocks - kb0) * q.x.le - m));
#pragma unroll
    for (int i = 0; i < IX; ++i) {
      const int row = (rq + i * (NW * 64 / GX)) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xc[i][j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (row + j) * int(q.x.ld) + gx * 8, 0, 0));
      xe[i] = __builtin_amdgcn_raw_buffer_load_b32(e, int(uint32_t(dkb) * uint32_t(q.x.le)) + row, 0, 0);
    }
  };
  const auto widen_x = [&](int64_t s, uint32_t stage) {
#pragma unroll
    for (int i = 0; i < IX; ++i) {
      const int row = (rq + i * (NW * 64 / GX)) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // rows past the last are zeros, whatever lies in place of their exponents
        const uint32_t byte = s * kSlice + row + j < q.M ? xe[i] >> (8 * j) & 0xffu : 127u;
        *reinterpret_cast<u32x4*>(ring + stage + kDy + (row + j) * TK * 2 + 16 * (gx ^ swz(row + j))) =
            values8(xc[i][j], byte);
      }
    }
  };

  f32x16 acc[NB][KB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < KB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  uint32_t cur = 0;
  if (s0 < s1) {
    issue_dy(s0, 0);
    load_x(s0);
    widen_x(s0, 0);
  }
  for (int64_t s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    const uint32_t next = kStage - cur;
    if (s + 1 < s1) {
      issue_dy(s + 1, next);
      load_x(s + 1);
    }
    const char* st = ring + cur;
#pragma unroll
    for (int c = 0; c < kSlice / 16; ++c) {
      bf16x8 fd[NB], fx[KB];
#pragma unroll
      for (int i = 0; i < NB; ++i) fd[i] = tr_frag<TN>(st, 16 * c, wn * 32 * NB + i * 32, lane);
#pragma unroll
      for (int j = 0; j < KB; ++j) fx[j] = tr_frag<TK>(st + kDy, 16 * c, wk * 32 * KB + j * 32, lane);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < KB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[i], fx[j], acc[i][j], 0, 0, 0);
    }
    if (s + 1 < s1) widen_x(s + 1, next);
    cur = next;
  }

  float* out = q.splits > 1 ? q.partial + int64_t(split) * q.N * q.K : q.dw;
  const int64_t ld = q.splits > 1 ? q.K : q.lddw;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      const int k = k0 + wk * 32 * KB + j * 32 + (lane & 31);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t n = n0 + wn * 32 * NB + i * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
        if (n < q.N && k < q.K) out[n * ld + k] = acc[i][j][r];
      }
    }
}

// The shares' sums, in order.
__global__ __launch_bounds__(256) void wgrad8_join_kernel(const WGrad8Params q) {
  const int g = q.K / 4;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= int64_t(q.N) * g) return;
  const int64_t n = i / g, k = i % g * 4;
  f32x4 v = *reinterpret_cast<const f32x4*>(q.partial + n * q.K + k);
  for (int s = 1; s < q.splits; ++s) v += *reinterpret_cast<const f32x4*>(q.partial + (int64_t(s) * q.N + n) * q.K + k);
  *reinterpret_cast<f32x4*>(q.dw + n * q.lddw + k) = v;
}

template <int NB, int KB, int WN, int WK>
void launch_tile(const WGrad8Params& q, hipStream_t s) {
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK;
  const int64_t tiles = int64_t((q.N + TN - 1) / TN) * ((q.K + TK - 1) / TK);
  hipLaunchKernelGGL((wgrad8_kernel<NB, KB, WN, WK>), dim3(tiles * q.splits), dim3(WN * WK * 64), 0, s, q);
}

}  // namespace

int launch_wgrad8(const WGrad8Params& q, int32_t tile, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (tile == 0) launch_tile<4, 2, 2, 4>(q, s);
  else launch_tile<2, 2, 2, 2>(q, s);
  if (q.splits > 1)
    hipLaunchKernelGGL(wgrad8_join_kernel, dim3((int64_t(q.N) * (q.K / 4) + 255) / 256), dim3(256), 0, s, q);
  return int(hipGetLastError());
}

}  // namespace rc
