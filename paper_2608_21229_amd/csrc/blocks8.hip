// Quantisation to e4m3 codes with one power-of-two scale per block of 128
// values, and back.
//
// A block's scale is 2^e with the smallest e >= -127 that brings its largest
// finite magnitude to at most 448, the largest e4m3 value; e = 0 for a block of
// zeros.  The code of x is the e4m3 value nearest to x 2^-e (ties to even):
// multiplying by a power of two is exact, so a code depends on its value and
// the block's maximum alone.  Infinities and NaN become the code of NaN.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_blocks8.h"
#include "rc_lds.h"
#include "rc_quant8.h"

namespace rc {
namespace {

// Blocks of a row.  A work-group takes kRows rows of four blocks: 16 lanes hold
// a block, 8 values each, so a wave reads 1 KB of a row at once, and all of a
// thread's rows are in flight together.  The exponents are gathered in LDS so
// that a block's column of them is written in runs of kRows bytes.
// Memory-bound: 2 bytes read and 1 written per value; 25 152 x 2560 takes 28.9 us
// (6.7 TB/s, partly from the last-level cache).  Loads by buffer descriptor: with a
// branch around each, the compiler waited for one at a time (47 us).
constexpr int kRows = 32;

__global__ __launch_bounds__(256) void quantize_rows_kernel(const Quant8Params q) {
  __shared__ uint8_t exps[4][kRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kblocks = (q.K + kBlock8 - 1) / kBlock8, groups = (kblocks + 3) / 4;
  const int64_t m0 = int64_t(blockIdx.x) / groups * kRows;
  const int kb0 = int(blockIdx.x % groups) * 4;
  const int kb = kb0 + (lane >> 4);
  const int64_t col = int64_t(kb0) * kBlock8 + lane * 8;
  const __amdgpu_buffer_rsrc_t x =
      bytes_rsrc(q.x + m0 * q.ldx, ((min(int64_t(kRows), q.M - m0) - 1) * q.ldx + q.K) * 2);
  u32x4 v[kRows / 4];
#pragma unroll
  for (int i = 0; i < kRows / 4; ++i) {
    v[i] = load16(x, uint32_t(i * 4 + wave) * uint32_t(q.ldx) * 2u + uint32_t(col) * 2u, col < q.K);
  }
  uint32_t top[kRows / 4];
  finite_abs_max(v, top);
#pragma unroll
  for (int i = 0; i < kRows / 4; ++i) {
    const int row = i * 4 + wave;
    const uint32_t byte = exponent_byte(group_max16(top[i]));
    if (m0 + row < q.M && kb < kblocks) *reinterpret_cast<u32x2*>(q.out.codes + (m0 + row) * q.out.ld + col) = codes8(v[i], byte);
    if ((lane & 15) == 0) exps[lane >> 4][row] = uint8_t(byte);
  }
  __syncthreads();
  if (threadIdx.x < 4 * kRows / 4) {
    const int k = threadIdx.x / (kRows / 4), r = threadIdx.x % (kRows / 4) * 4;
    if (kb0 + k < kblocks && m0 + r < q.out.le)
      *reinterpret_cast<uint32_t*>(q.out.exps + int64_t(kb0 + k) * q.out.le + m0 + r) =
          *reinterpret_cast<const uint32_t*>(&exps[k][r]);
  }
}

// 4 x 4 bytes, rows to columns.
__device__ __forceinline__ void transpose4(uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, uint32_t (&c)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(r1, r0, 0x05010400u), b = __builtin_amdgcn_perm(r1, r0, 0x07030602u);
  const uint32_t d = __builtin_amdgcn_perm(r3, r2, 0x05010400u), e = __builtin_amdgcn_perm(r3, r2, 0x07030602u);
  c[0] = __builtin_amdgcn_perm(d, a, 0x05040100u);
  c[1] = __builtin_amdgcn_perm(d, a, 0x07060302u);
  c[2] = __builtin_amdgcn_perm(e, b, 0x05040100u);
  c[3] = __builtin_amdgcn_perm(e, b, 0x07060302u);
}

// Squares of 128 x 128, one per work-group, 8 x 8 values per thread, whose
// codes are transposed in registers; LDS only gathers them into whole rows (8-byte
// part p of row k at part p ^ (k / 8)).  Columns up to the next multiple of 128 exist
// as zeros.  Memory-bound: 2 bytes read and 1 or 2 written per value; 7680 x 2560
// with the transposed form takes 12.7 us (6.2 TB/s; with bytes gathered from LDS 19).
__global__ __launch_bounds__(256) void quantize_squares_kernel(const Quant8Params q) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock8 * kBlock8];
  __shared__ uint32_t red[4];
  const int t = threadIdx.x, c8 = t & 15, r8 = t >> 4;
  const int kblocks = (q.K + kBlock8 - 1) / kBlock8;
  const int64_t nb = int64_t(blockIdx.x) / kblocks;
  const int kb = int(blockIdx.x % kblocks);
  const int64_t m0 = nb * kBlock8, k0 = int64_t(kb) * kBlock8;
  const int64_t col = k0 + c8 * 8, row = m0 + r8 * 8;
  const __amdgpu_buffer_rsrc_t x =
      bytes_rsrc(q.x + m0 * q.ldx, ((min(int64_t(kBlock8), q.M - m0) - 1) * q.ldx + q.K) * 2);
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = load16(x, uint32_t(r8 * 8 + i) * uint32_t(q.ldx) * 2u + uint32_t(col) * 2u, col < q.K);
  }
  uint32_t a = finite_abs_max(v);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) a = max(a, uint32_t(__shfl_xor(int(a), s)));
  if ((t & 63) == 0) red[t >> 6] = a;
  __syncthreads();
  const uint32_t byte = exponent_byte(max(max(red[0], red[1]), max(red[2], red[3])));
  u32x2 c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = codes8(v[i], byte);
    if (row + i < q.M) *reinterpret_cast<u32x2*>(q.out.codes + (row + i) * q.out.ld + col) = c[i];
  }
  const uint32_t four = byte * 0x01010101u;
  if (t < 32) {
    if (m0 + t * 4 < q.out.le) *reinterpret_cast<uint32_t*>(q.out.exps + kb * q.out.le + m0 + t * 4) = four;
  } else if (t < 64 && q.out_t.codes) {
    const int r = (t - 32) * 4;
    if (k0 + r < q.out_t.le) *reinterpret_cast<uint32_t*>(q.out_t.exps + nb * q.out_t.le + k0 + r) = four;
  }
  if (!q.out_t.codes) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t lo[4], hi[4];
    transpose4(c[0][h], c[1][h], c[2][h], c[3][h], lo);
    transpose4(c[4][h], c[5][h], c[6][h], c[7][h], hi);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<u32x2*>(tile + (c8 * 8 + 4 * h + e) * kBlock8 + (r8 ^ c8) * 8) = u32x2{lo[e], hi[e]};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = i * 16 + (t >> 4), n8 = t & 15;
    if (k0 + k < q.K)
      *reinterpret_cast<u32x2*>(q.out_t.codes + (k0 + k) * q.out_t.ld + m0 + n8 * 8) =
          *reinterpret_cast<const u32x2*>(tile + k * kBlock8 + (n8 ^ (k >> 3)) * 8);
  }
}

// 8 codes per thread back to bf16, exact (4 significant bits) above bf16's smallest; the
// largest code of the largest scale, 2^128, is infinite.
// Memory-bound: 25 152 x 2560 takes 30 us (6.4 TB/s).
__global__ __launch_bounds__(256) void dequantize_kernel(const Dequant8Params q) {
  const int g = q.K / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= q.M * g) return;
  const int64_t m = i / g;
  const int col = int(i % g) * 8;
  const u32x2 c = *reinterpret_cast<const u32x2*>(q.x.codes + m * q.x.ld + col);
  *reinterpret_cast<u32x4*>(q.out + m * q.ldo + col) = values8(c, q.x.exps[int64_t(col / kBlock8) * q.x.le + m]);
}

}  // namespace

int launch_quantize_rows(const Quant8Params& q, void* stream) {
  const int64_t groups = (blocks8(q.K) + 3) / 4;
  hipLaunchKernelGGL(quantize_rows_kernel, dim3((q.M + kRows - 1) / kRows * groups), dim3(256), 0,
                     static_cast<hipStream_t>(stream), q);
  return int(hipGetLastError());
}

int launch_quantize_squares(const Quant8Params& q, void* stream) {
  hipLaunchKernelGGL(quantize_squares_kernel, dim3(blocks8(q.M) * blocks8(q.K)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), q);
  return int(hipGetLastError());
}

int launch_dequantize(const Dequant8Params& q, void* stream) {
  hipLaunchKernelGGL(dequantize_kernel, dim3((q.M * (q.K / 8) + 255) / 256), dim3(256), 0,
                     static_cast<hipStream_t>(stream), q);
  return int(hipGetLastError());
}

}  // namespace rc
