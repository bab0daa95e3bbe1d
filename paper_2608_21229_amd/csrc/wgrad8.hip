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

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr int kSlice = 64;  // rows per step

// Granule g (8 columns) of row r lies at slot g ^ swz(r): the four rows of a
// transpose read fall into four quarters of the banks.
__device__ __forceinline__ int swz(int row) { return (row & 3) << 2 | (row >> 2 & 3); }

// Tiles of n x k: WN x WK waves, each NB x KB accumulators of 32 x 32, one wave
// per SIMD.  The first `whole` work-groups take a tile each, with all rows; the
// remaining tiles, less than a round of the CUs, are cut into `splits` shares of
// their rows, whose sums go to the workspace and are added in order by the join.
// Shares of the same rows are neighbours on one XCD: they read the same dy and x
// from its L2 (250 shares in another order were bound by 7.8 TB/s of them).
//
// A ring of ST stages of 64 rows of both operands.  A wave runs one stream of
// matrix instructions; between them, in an order fixed by scheduling fences, go
// the fragment reads of the next 16 rows, the widening of the next slice's codes
// (loaded into one of XD sets of registers XD slices ago, then reloaded) and the
// direct loads of dy.  The one barrier per slice lies before its last 16 rows,
// whose fragments are in registers by then: behind it the next slice's first
// fragments are read, and dy of the slice ST further is loaded into the stage that
// has just been read.  A smaller tile has less time per slice, so its loads go out
// more slices ahead.  Slices past the share's last one load zeros, so the loop has
// no other branch, and runs a multiple of XD slices.
template <int NB, int KB, int WN, int WK, int ST, int XD>
__global__ __launch_bounds__(WN * WK * 64) __attribute__((amdgpu_waves_per_eu(1, 1))) void wgrad8_kernel(
    const WGrad8Params q) {
  constexpr int NW = WN * WK;
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK;
  constexpr int kDy = kSlice * TN * 2, kX = kSlice * TK * 2, kStage = kDy + kX;
  constexpr int CD = kDy / 1024 / NW;            // 1 KB chunks of dy per wave
  constexpr int GX = TK / 8;                     // granules of a row of x
  constexpr int RQ = kSlice / 4;                 // groups of four rows
  constexpr int IX = RQ * GX / (NW * 64);        // groups per thread
  constexpr int NX = IX * 4;                     // granules per thread
  static_assert(CD * NW * 1024 == kDy && IX * NW * 64 == RQ * GX && NW * 64 % GX == 0, "loads divide over the waves");
  __shared__ __attribute__((aligned(1024))) char ring[ST * kStage];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave / WK, wk = wave % WK;

  const int64_t rows_n = (q.N + TN - 1) / TN, cols_k = (q.K + TK - 1) / TK, tiles = rows_n * cols_k;
  int64_t tile, share = -1;
  if (int64_t(blockIdx.x) < q.whole) {
    tile = xcd_block(blockIdx.x, q.whole);
  } else {
    const int64_t rest = tiles - q.whole;
    share = xcd_block(blockIdx.x - q.whole, rest * q.splits);
    tile = q.whole + share % rest;
  }
  int64_t tn, tk;
  grouped_tile(tile, rows_n, cols_k, 4, tn, tk);
  const int n0 = int(tn * TN), k0 = int(tk * TK);
  const int64_t slices = (q.M + kSlice - 1) / kSlice;
  int64_t s0 = 0, s1 = slices;
  if (share >= 0) {
    const int64_t split = share / (tiles - q.whole);
    s0 = slices * split / q.splits;
    s1 = slices * (split + 1) / q.splits;
  }

  // dy: lane l of chunk c fills slot 64 c + l
  constexpr int GD = TN / 8;
  uint32_t doff[CD];
#pragma unroll
  for (int i = 0; i < CD; ++i) {
    const int p = (i * NW + wave) * 64 + lane, row = p / GD;
    doff[i] = uint32_t(row) * uint32_t(q.lddy) * 2u + uint32_t((p % GD) ^ swz(row)) * 16u;
  }
  const uint32_t lds0 = lds_u32(ring);
  const auto issue_dy = [&](uint32_t stage, __amdgpu_buffer_rsrc_t r, int i) {
    dma16(lds0 + stage + uint32_t((i * NW + wave) * 1024), doff[i], r);
  };

  // x: a thread takes 8 codes of four consecutive rows, whose exponents are one
  // dword, IX times; granule j of a slice is in xc[j]
  const int gx = tid % GX, xrow = tid / GX * 4;
  constexpr int kRowStep = NW * 64 / GX * 4;  // rows between a thread's groups
  const int kblocks = int(blocks8(q.K)), kb0 = k0 / kBlock8;
  const int dkb = min(gx * 8 / kBlock8, kblocks - 1 - kb0);
  u32x2 xc[XD][NX];
  uint32_t xe[XD][IX], xe_now = 0;
  int xoff[NX], eoff[IX];
#pragma unroll
  for (int j = 0; j < NX; ++j) xoff[j] = (xrow + j / 4 * kRowStep + j % 4) * int(q.x.ld) + gx * 8;
#pragma unroll
  for (int i = 0; i < IX; ++i) eoff[i] = int(uint32_t(dkb) * uint32_t(q.x.le)) + xrow + i * kRowStep;
  const auto load_codes = [&](int set, __amdgpu_buffer_rsrc_t r, int j) {
    xc[set][j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, xoff[j], 0, 0));
  };
  const auto load_exps = [&](int set, __amdgpu_buffer_rsrc_t r, int i) {
    xe[set][i] = __builtin_amdgcn_raw_buffer_load_b32(r, eoff[i], 0, 0);
  };
  static_assert(kRowStep % 16 == 0, "a thread's groups have one swizzle");
  uint32_t xlds[4];  // where the granules of a group go
#pragma unroll
  for (int j = 0; j < 4; ++j) xlds[j] = uint32_t(kDy + (xrow + j) * TK * 2 + 16 * (gx ^ swz(xrow + j)));
  // granule j with the exponents of its group in xe_now
  const auto widen = [&](int set, uint32_t stage, int j) {
    *reinterpret_cast<u32x4*>(ring + stage + xlds[j % 4] + j / 4 * kRowStep * TK * 2) =
        values8_any(xc[set][j], xe_now >> (8 * (j % 4)));
  };

  // The streams of slices: where the next one starts and the share's rows from
  // there on.  Loads past the rows (and of slices past the last) give zeros.
  const int64_t m0 = s0 * kSlice;
  const int rows = int(min(s1 * kSlice, q.M) - m0);
  const char* dy_at = reinterpret_cast<const char*>(q.dy + m0 * q.lddy + n0);
  const uint8_t* codes_at = q.x.codes + m0 * q.x.ld + k0;
  const uint8_t* exps_at = q.x.exps + kb0 * q.x.le + m0;
  int dy_left = rows, codes_left = rows;
  const int dy_cols = min(TN, q.N - n0) * 2, x_cols = min(TK, kblocks * kBlock8 - k0);
  const int dy_ld = int(q.lddy) * 2, x_ld = int(q.x.ld);
  const int64_t exps_more = (kblocks - kb0) * q.x.le - m0;
  const auto next_dy = [&] {
    const __amdgpu_buffer_rsrc_t r = bytes_rsrc(dy_at, dy_left > 0 ? (min(kSlice, dy_left) - 1) * dy_ld + dy_cols : 0);
    dy_at += kSlice * dy_ld;
    dy_left -= kSlice;
    return r;
  };
  // the codes' descriptor, then the exponents'
  const auto next_codes = [&] {
    return bytes_rsrc(codes_at, codes_left > 0 ? (min(kSlice, codes_left) - 1) * x_ld + x_cols : 0);
  };
  uint32_t exps_size = uint32_t(min(int64_t(0x7fffffff), exps_more));
  const bool exps_cut = exps_more > 0x7fffffff;
  const auto next_exps = [&] {
    const __amdgpu_buffer_rsrc_t r = bytes_rsrc(exps_at, codes_left > 0 ? exps_size : 0);
    codes_at += kSlice * x_ld;
    exps_at += kSlice;
    codes_left -= kSlice;
    if (!exps_cut) exps_size -= kSlice;
    return r;
  };

  // fragment addresses: a lane's granule in block f, and 8 rows further; slices
  // of 16 rows are constants
  const int li = lane & 15, r0 = 4 * (lane >> 5) + (li >> 2), g0 = 2 * (lane >> 4 & 1) + ((li & 3) >> 1);
  constexpr int NF = NB + KB, NM = NB * KB;
  uint32_t fa[NF][2];
#pragma unroll
  for (int t = 0; t < NF; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int columns = t < NB ? TN : TK, c0 = t < NB ? wn * 32 * NB + t * 32 : wk * 32 * KB + (t - NB) * 32;
      const int row = r0 + 8 * h;
      fa[t][h] = lds0 + (t < NB ? 0 : kDy) + row * columns * 2 + 16 * ((c0 / 8 + g0) ^ swz(row)) + 8 * (li & 1);
    }
  i16x4 fr[2][NF][2];
  // half h of fragment t of 16-row chunk c
  const auto read = [&](int c, int t, int h) {
    fr[c % 2][t][h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)uintptr_t(fa[t][h] + 16 * c * (t < NB ? TN : TK) * 2));
  };
  const auto frag = [&](int c, int t) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(fr[c % 2][t][0], fr[c % 2][t][1], 0, 1, 2, 3, 4, 5, 6, 7));
  };

  f32x16 acc[NB][KB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < KB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  constexpr int kNewer = (ST - 2) * (CD + NX + IX) + NX + IX;  // loads behind those of the next slice's dy
  static_assert(kNewer <= 63, "vmcnt range");
  const int n_slices = int(s1 - s0);
  __amdgpu_buffer_rsrc_t r_codes, r_exps;
  if (n_slices > 0) {
    // in the order in which the loop reloads them
    const auto load_x = [&](int set) {
      r_codes = next_codes();
      r_exps = next_exps();
#pragma unroll
      for (int j = 0; j < NX; ++j) {
        if (j % 4 == 0) load_exps(set, r_exps, j / 4);
        sched_fence();
        load_codes(set, r_codes, j);
        sched_fence();
      }
    };
    load_x(0);
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const __amdgpu_buffer_rsrc_t r = next_dy();
#pragma unroll
      for (int i = 0; i < CD; ++i) issue_dy(s * kStage, r, i);
    }
#pragma unroll
    for (int j = 0; j < NX; ++j) {
      xe_now = xe[0][j / 4];
      widen(0, 0, j);
    }
#pragma unroll
    for (int x = 1; x <= XD; ++x) load_x(x % XD);
    r_codes = next_codes();
    r_exps = next_exps();
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(XD * (NX + IX)) : "memory");
    lds_barrier();
#pragma unroll
    for (int t = 0; t < NF; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) read(0, t, h);
  }
  uint32_t cur = 0;
  // slice s, whose successor's codes are in `set`
  const auto slice = [&](int set) {
    const uint32_t next = cur + kStage == ST * kStage ? 0 : cur + kStage;
    __amdgpu_buffer_rsrc_t r_dy;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c == 3) {
        // dy of the next slice has landed, its x is written
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kNewer) : "memory");
        lds_barrier();
      }
#pragma unroll
      for (int t = 0; t < NM; ++t) {
        // rows of the block are k, columns n: a lane's accumulator is of one row of dw
        acc[t / KB][t % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(c, NB + t % KB), frag(c, t / KB),
                                                                      acc[t / KB][t % KB], 0, 0, 0);
#pragma unroll
        for (int f = 0; f < 2 * NF; ++f)
          if (f * NM / (2 * NF) == t) {
            if (c == 3) fa[f / 2][f % 2] += next - cur;
            read((c + 1) % 4, f / 2, f % 2);
          }
        if (c == 3) {
#pragma unroll
          for (int i = 0; i < CD; ++i)
            if (i * NM / CD == t) issue_dy(cur, r_dy, i);
          if (t == NM / 2) r_codes = next_codes();
          if (t == NM - 1) r_exps = next_exps();
        } else {
#pragma unroll
          for (int j = 0; j < NX; ++j)
            if (j * 3 * NM / NX == c * NM + t) {
              if (j % 4 == 0) {
                xe_now = xe[set][j / 4];
                load_exps(set, r_exps, j / 4);
              }
              widen(set, next, j);
              load_codes(set, r_codes, j);
            }
          if (c == 2 && t == NM - 1) r_dy = next_dy();
        }
        sched_fence();
      }
    }
    cur = next;
  };
  for (int s = 0; s < n_slices; s += XD)
#pragma unroll
    for (int x = 1; x <= XD; ++x) slice(x % XD);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the work-group

  if (share >= 0 && q.splits > 1) {
    f32x4* out = reinterpret_cast<f32x4*>(q.partial) + share * (TN * TK / 4) + tid;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          out[((i * KB + j) * 4 + r) * (NW * 64)] =
              f32x4{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int64_t n = n0 + wn * 32 * NB + i * 32 + (lane & 31);
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = k0 + wk * 32 * KB + j * 32 + 8 * r + 4 * (lane >> 5);
          if (n < q.N && k < q.K)
            *reinterpret_cast<f32x4*>(q.dw + n * q.lddw + k) =
                f32x4{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
        }
    }
  }
}

// A work-group adds, in the order of the shares, one row of a tile's accumulator
// blocks (the same 32 x 32 block of every wave).
template <int NB, int KB, int WN, int WK>
__global__ __launch_bounds__(WN * WK * 64) void wgrad8_join_kernel(const WGrad8Params q) {
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK, kBlocks = NB * KB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wn = wave / WK, wk = wave % WK;
  const int64_t rows_n = (q.N + TN - 1) / TN, cols_k = (q.K + TK - 1) / TK, tiles = rows_n * cols_k;
  const int64_t rest = tiles - q.whole, t = int64_t(blockIdx.x) / kBlocks;
  const int block = int(blockIdx.x % kBlocks), i = block / KB, j = block % KB;
  f32x4 v[4] = {};
  for (int s = 0; s < q.splits; ++s) {
    const f32x4* in = reinterpret_cast<const f32x4*>(q.partial) + (s * rest + t) * (TN * TK / 4) + tid;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] += in[(block * 4 + r) * (WN * WK * 64)];
  }
  int64_t tn, tk;
  grouped_tile(q.whole + t, rows_n, cols_k, 4, tn, tk);
  const int64_t n = tn * TN + wn * 32 * NB + i * 32 + (lane & 31);
  const int64_t k = tk * TK + wk * 32 * KB + j * 32 + 4 * (lane >> 5);
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n < q.N && k + 8 * r < q.K) *reinterpret_cast<f32x4*>(q.dw + n * q.lddw + k + 8 * r) = v[r];
}

template <int NB, int KB, int WN, int WK, int ST, int XD>
void launch_tile(const WGrad8Params& q, hipStream_t s) {
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK;
  const int64_t rest = int64_t((q.N + TN - 1) / TN) * ((q.K + TK - 1) / TK) - q.whole;
  hipLaunchKernelGGL((wgrad8_kernel<NB, KB, WN, WK, ST, XD>), dim3(q.whole + rest * q.splits), dim3(WN * WK * 64), 0, s, q);
  if (q.splits > 1)
    hipLaunchKernelGGL((wgrad8_join_kernel<NB, KB, WN, WK>), dim3(rest * NB * KB), dim3(WN * WK * 64), 0, s, q);
}

}  // namespace

int launch_wgrad8(const WGrad8Params& q, int32_t tile, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (tile) {
    case 0: launch_tile<4, 4, 2, 2, 2, 1>(q, s); break;
    case 1: launch_tile<4, 2, 2, 2, 3, 2>(q, s); break;
    default: launch_tile<2, 2, 2, 2, 4, 2>(q, s); break;
  }
  return int(hipGetLastError());
}

}  // namespace rc
