// Gradient of a projection's weights from an 8-bit checkpoint of its input:
//
//   dw[n, k] = sum_m dy[m, n] x[m, k],  x = code 2^e, dy in bf16, fp32 sums and result
//
// The codes are widened to bf16 (exact below 2^128), so the product is one of
// v_mfma_f32_32x32x16_bf16.  The sum runs over rows, which both operands hold as
// their slow dimension; they are transposed in registers on their way into LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_blocks8.h"
#include "rc_lds.h"
#include "rc_quant8.h"

namespace rc {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(3))) bf16x8 lds_cbf16x8;

constexpr int kSlice = 64;  // rows per step

// LDS holds a slice's columns as rows of 64 values (128 bytes); the 16 bytes of 8
// rows g of column c lie at part g ^ part8(c): the writes, of columns 4 or 8 apart,
// and the reads, of neighbouring columns, both meet every bank once.
__device__ __forceinline__ int part8(int c) { return (c ^ c >> 3) & 7; }

// 4 or 8 columns of 8 rows, as loaded: row r's are in d[r].
template <int P>
struct Block {
  uint32_t d[8][P / 4];  // codes
};
template <int P>
struct BlockBf16 {
  uint32_t d[8][P / 2];
};

// The 16 bytes of column 2 p (or 2 p + 1) of 8 rows, of whose dwords each holds both.
template <bool ODD>
__device__ __forceinline__ u32x4 column(const uint32_t (&r)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(r[2 * i + 1], r[2 * i], ODD ? 0x07060302u : 0x05040100u);
  return v;
}

// Tiles of n x k: WN x WK waves, each NB x KB accumulators of 32 x 32, one wave
// per SIMD.  The first `whole` work-groups take a tile each, with all rows; the
// remaining tiles, less than a round of the CUs, are cut into `splits` shares of
// their rows, whose sums go to the workspace and are added in order by the join.
// Shares of the same rows are neighbours on one XCD: they read the same dy and x
// from its L2.
//
// Two stages of 64 rows of both operands.  A wave runs one stream of matrix
// instructions; between them, in an order fixed by scheduling fences, go the
// fragment reads of the next 16 rows and the way of the slices ahead: a thread
// holds 8 rows of 4 or 8 columns of each operand in registers, widens and transposes
// them into the stage that is free, and loads the next slice's.  The one barrier per
// slice lies before its last 16 rows, whose fragments are in registers by then:
// behind it the next slice's first fragments are read, and its own stage is written
// again.  Slices past the share's last one load zeros, so the loop has no other branch.
//
// What bounds it (256 x 256): 64 products of 32 cycles per slice and SIMD, 2048, and the
// issue of what goes between them.  On 25 tiles, at 2.42 GHz, a slice takes 2 980 cycles
// (counters: LDS busy 1 030 of them, waits 380, the rest waits for issue); on a full
// chip, whose clock falls, 1.6 us: 17 536 x 4096 x 4096 runs in 439-460 us (1.28-1.34
// PFLOP/s; the library's 8192 cubed reaches 1.43).  17 536 x 7680 x 2560, 300 tiles, takes
// 558-579 us with its join (the library's product of transposed dy 912).  Forms measured before, at these
// two: dy loaded straight into LDS and both operands read by the transpose read
// ds_read_b64_tr_b16, 443 and 591 us; both transposed in registers with one slice there,
// 477 and 596; with two, 463 and 573 until the pieces behind a product became as short
// as it hides.  On few tiles, a slice of the smaller ones takes 0.79 us (256 x 128) and
// 0.63 (128 x 128).
template <int NB, int KB, int WN, int WK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void wgrad8_kernel(const WGrad8Params q) {
  static_assert(WN * WK == 4, "four waves");
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK, PN = TN / 32, PK = TK / 32;
  constexpr int kDy = kSlice * TN * 2, kX = kSlice * TK * 2, kStage = kDy + kX;
  __shared__ __attribute__((aligned(1024))) char ring[2 * kStage];
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

  // This thread's 8 rows and its columns of both operands.
  const int col = tid & 31, row8 = tid >> 5;
  const int kblocks = int(blocks8(q.K)), kb0 = k0 / kBlock8;
  const int dkb = min(col * PK / kBlock8, kblocks - 1 - kb0);
  const int64_t m0 = s0 * kSlice;
  const int rows = int(min(s1 * kSlice, q.M) - m0);
  // The streams of slices: where the next one starts and the share's rows from
  // there on.  Loads past the rows (and of slices past the last) give zeros.
  const char* dy_at = reinterpret_cast<const char*>(q.dy + m0 * q.lddy + n0);
  const uint8_t* codes_at = q.x.codes + m0 * q.x.ld + k0;
  const uint8_t* exps_at = q.x.exps + kb0 * q.x.le + m0;
  int dy_left = rows, codes_left = rows;
  const int dy_cols = min(TN, q.N - n0) * 2, x_cols = min(TK, kblocks * kBlock8 - k0);
  const int dy_ld = int(q.lddy) * 2, x_ld = int(q.x.ld);
  const int64_t exps_more = (kblocks - kb0) * q.x.le - m0;
  uint32_t exps_size = uint32_t(min(int64_t(0x7fffffff), exps_more));
  const bool exps_cut = exps_more > 0x7fffffff;
  __amdgpu_buffer_rsrc_t r_dy, r_codes, r_exps;
  const auto next_dy = [&] {
    r_dy = bytes_rsrc(dy_at, max(0, min(kSlice, dy_left) * dy_ld - (dy_ld - dy_cols)));
    dy_at += kSlice * dy_ld;
    dy_left -= kSlice;
  };
  const auto next_codes = [&] {
    r_codes = bytes_rsrc(codes_at, max(0, min(kSlice, codes_left) * x_ld - (x_ld - x_cols)));
    codes_at += kSlice * x_ld;
  };
  const auto next_exps = [&] {
    r_exps = bytes_rsrc(exps_at, codes_left > 0 ? exps_size : 0);
    exps_at += kSlice;
    codes_left -= kSlice;
    if (!exps_cut) exps_size -= kSlice;
  };
  // two slices of each, and the exponents of their 8 rows
  BlockBf16<PN> dy[2];
  Block<PK> x[2];
  u32x2 xe[2];
  const uint32_t dy_off = uint32_t(row8 * 8) * uint32_t(dy_ld) + uint32_t(col * PN * 2);
  const uint32_t x_off = uint32_t(row8 * 8) * uint32_t(x_ld) + uint32_t(col * PK);
  const uint32_t e_off = uint32_t(dkb) * uint32_t(q.x.le) + uint32_t(row8 * 8);
  const auto load_dy = [&](int set, int r) {
    const int at = int(dy_off + uint32_t(r) * uint32_t(dy_ld));
    if constexpr (PN == 8) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r_dy, at, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) dy[set].d[r][i] = v[i];
    } else {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r_dy, at, 0, 0);
      dy[set].d[r][0] = v[0];
      dy[set].d[r][1] = v[1];
    }
  };
  const auto load_codes = [&](int set, int r) {
    const int at = int(x_off + uint32_t(r) * uint32_t(x_ld));
    if constexpr (PK == 8) {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r_codes, at, 0, 0);
      x[set].d[r][0] = v[0];
      x[set].d[r][1] = v[1];
    } else {
      x[set].d[r][0] = __builtin_amdgcn_raw_buffer_load_b32(r_codes, at, 0, 0);
    }
  };
  const auto load_exps = [&](int set) { xe[set] = __builtin_amdgcn_raw_buffer_load_b64(r_exps, int(e_off), 0, 0); };

  // A slice's way to LDS in pieces of a few instructions, one or two of which go
  // behind a product (32 cycles, which hide about seven): a column of dy; of x two
  // columns, in four pieces: half of the rows widened, the others, each column written.
  const auto put = [&](uint32_t at, int c, u32x4 v) {
    *reinterpret_cast<u32x4*>(ring + at + c * (kSlice * 2) + 16 * (row8 ^ part8(c))) = v;
  };
  const auto put_dy = [&](int set, uint32_t stage, int c) {
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = dy[set].d[i][c / 2];
    put(stage, col * PN + c, c % 2 ? column<true>(r) : column<false>(r));
  };
  float scale[8];
  uint32_t wide[8];
  const auto take_scale = [&](int set, int i) { scale[i] = scale8_any(xe[set][i / 4] >> (8 * (i % 4))); };
  const auto put_x = [&](int set, uint32_t stage, int piece) {
    const int p = piece / 4, part = piece % 4;
    if (part < 2) {
#pragma unroll
      for (int i = 4 * part; i < 4 * part + 4; ++i)
        wide[i] = p % 2 ? widened<true>(x[set].d[i][p / 2], scale[i]) : widened<false>(x[set].d[i][p / 2], scale[i]);
    } else {
      put(stage + kDy, col * PK + 2 * p + part - 2, part == 3 ? column<true>(wide) : column<false>(wide));
    }
  };

  // Fragments: columns c0 + lane % 32, rows 16 c + 8 (lane / 32) ..  of a slice.  Of
  // block f of an operand the part differs in bit 2, of rows 16 c in bits 1 and 2.
  constexpr int NF = NB + KB, NM = NB * KB;
  const uint32_t lds0 = lds_u32(ring);
  uint32_t fa[2];
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int c = (o == 0 ? wn * 32 * NB : wk * 32 * KB) + (lane & 31);
    fa[o] = lds0 + (o == 0 ? 0 : kDy) + c * (kSlice * 2) + 16 * ((lane >> 5) ^ part8(c));
  }
  bf16x8 fr[2][NF];
  const auto read = [&](int c, int t) {
    const int o = t < NB ? 0 : 1, f = t < NB ? t : t - NB;
    fr[c % 2][t] = *(lds_cbf16x8*)uintptr_t((fa[o] ^ uint32_t(32 * c) ^ uint32_t(64 * (f & 1))) + f * 32 * kSlice * 2);
  };

  f32x16 acc[NB][KB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < KB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const int n_slices = int(s1 - s0);
  if (n_slices > 0) {
    // slices 0, 1 and 2 of the share, the last two of which stay in the registers
    // (the second one's x is written: the loop takes its dy)
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      next_codes();
      next_exps();
      next_dy();
      load_exps(s % 2);
#pragma unroll
      for (int r = 0; r < 8; ++r) load_codes(s % 2, r);
#pragma unroll
      for (int r = 0; r < 8; ++r) load_dy(s % 2, r);
      if (s == 2) break;
#pragma unroll
      for (int i = 0; i < 8; ++i) take_scale(s, i);
#pragma unroll
      for (int p = 0; p < 2 * PK; ++p) put_x(s, s * kStage, p);
      if (s == 0)
#pragma unroll
        for (int c = 0; c < PN; ++c) put_dy(0, 0, c);
    }
    next_codes();
    next_exps();
    next_dy();
    lds_barrier();
#pragma unroll
    for (int t = 0; t < NF; ++t) read(0, t);
  }
  // Slice s, in stage and register set s % 2.
  const auto slice = [&](int set) {
    const uint32_t cur = set * kStage, next = kStage - cur;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c == 3) lds_barrier();
#pragma unroll
      for (int t = 0; t < NM; ++t) {
        // rows of the block are k, columns n: a lane's accumulator is of one row of dw
        acc[t / KB][t % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[c % 2][NB + t % KB], fr[c % 2][t / KB],
                                                                      acc[t / KB][t % KB], 0, 0, 0);
#pragma unroll
        for (int f = 0; f < NF; ++f)
          if (f * NM / NF == t) read((c + 1) % 4, f);
        if (c == 0) {  // dy of slice s + 1 to LDS, x of slice s + 3 to its registers
#pragma unroll
          for (int p = 0; p < PN; ++p)
            if (p * NM / PN == t) put_dy(1 - set, next, p);
          if (t == 0) load_exps(1 - set);
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (r * NM / 8 == t) load_codes(1 - set, r);
        }
        if (c == 1) {  // dy of slice s + 3
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (r * NM / 8 == t) load_dy(1 - set, r);
        }
        if (c == 2) {
          if (t == 0) next_codes();
          if (t == NM / 4) next_exps();
          if (t == NM / 2) next_dy();
          if (t == NM - 1) fa[0] += next - cur, fa[1] += next - cur;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i * NM / 8 == t) take_scale(set, i);
        }
        if (c == 3) {  // x of slice s + 2, into the stage that has been read
#pragma unroll
          for (int p = 0; p < 2 * PK; ++p)
            if (p * NM / (2 * PK) == t) put_x(set, cur, p);
        }
        sched_fence();
      }
    }
  };
  for (int s = 0; s + 1 < n_slices; s += 2) {
    slice(0);
    slice(1);
  }
  if (n_slices & 1) slice(0);

  if (share >= 0 && q.splits > 1) {
    f32x4* out = reinterpret_cast<f32x4*>(q.partial) + share * (TN * TK / 4) + tid;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          out[((i * KB + j) * 4 + r) * 256] =
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

// A work-group adds, in the order of the shares, a quarter of a tile's accumulator
// blocks (i, j) of every wave, four shares' loads in flight.
template <int NB, int KB, int WN, int WK>
__global__ __launch_bounds__(256) void wgrad8_join_kernel(const WGrad8Params q) {
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK, kParts = NB * KB * 4, kAhead = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wn = wave / WK, wk = wave % WK;
  const int64_t rows_n = (q.N + TN - 1) / TN, cols_k = (q.K + TK - 1) / TK;
  const int64_t rest = rows_n * cols_k - q.whole, t = int64_t(blockIdx.x) / kParts;
  const int part = int(blockIdx.x % kParts), i = part / 4 / KB, j = part / 4 % KB;
  const f32x4* in = reinterpret_cast<const f32x4*>(q.partial) + t * (TN * TK / 4) + part * 256 + tid;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < q.splits; s += kAhead) {
    f32x4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = in[min(s + u, q.splits - 1) * rest * (TN * TK / 4)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s + u < q.splits) v += w[u];
  }
  int64_t tn, tk;
  grouped_tile(q.whole + t, rows_n, cols_k, 4, tn, tk);
  const int64_t n = tn * TN + wn * 32 * NB + i * 32 + (lane & 31);
  const int64_t k = tk * TK + wk * 32 * KB + j * 32 + 4 * (lane >> 5) + part % 4 * 8;
  if (n < q.N && k < q.K) *reinterpret_cast<f32x4*>(q.dw + n * q.lddw + k) = v;
}

template <int NB, int KB, int WN, int WK>
void launch_tile(const WGrad8Params& q, hipStream_t s) {
  constexpr int TN = 32 * NB * WN, TK = 32 * KB * WK;
  const int64_t rest = int64_t((q.N + TN - 1) / TN) * ((q.K + TK - 1) / TK) - q.whole;
  hipLaunchKernelGGL((wgrad8_kernel<NB, KB, WN, WK>), dim3(q.whole + rest * q.splits), dim3(WN * WK * 64), 0, s, q);
  if (q.splits > 1)
    hipLaunchKernelGGL((wgrad8_join_kernel<NB, KB, WN, WK>), dim3(rest * NB * KB * 4), dim3(256), 0, s, q);
}

}  // namespace

int launch_wgrad8(const WGrad8Params& q, int32_t tile, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (tile) {
    case 0: launch_tile<4, 4, 2, 2>(q, s); break;
    case 1: launch_tile<4, 2, 2, 2>(q, s); break;
    default: launch_tile<2, 2, 2, 2>(q, s); break;
  }
  return int(hipGetLastError());
}

}  // namespace rc
