// Projection of e4m3 blocks: out = a W^T (+ r), both operands codes with one
// power-of-two scale per 128 values of a row.
//
//   out[m, n] = bf16( sum_kb 2^(ea[m, kb] + ew[n, kb]) sum_{k in kb} a[m, k] w[n, k]  (+ r[m, n]) )
//
// The scaled matrix instructions (v_mfma_scale_f32_*_f8f6f4) take the exponents
// as operands, one byte per row and 32 values, so the scaling costs nothing and
// the sums stay in one fp32 accumulator over all of k.  What they round (found with
// cancelling products): each of a group of eight neighbouring products is cut,
// towards zero, to a multiple of 2^-13 of the largest power of two among them, the
// product of those in both codes (2^-6 for subnormal ones) and both scales; sums
// beyond that are fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_blocks8.h"
#include "rc_lds.h"
#include "rc_quant8.h"

namespace rc {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

constexpr int kBK = kBlock8;     // codes of a row per slice: one 128-byte LDS row, one scale
constexpr int kScaleSlices = 8;  // slices whose scales are loaded together

// 16-byte granule g of row r lies at slot g ^ ((r >> 1) & 7), so that the reads
// of 16 consecutive rows hit 16 distinct bank groups.
__device__ __forceinline__ int slot8(int row, int g) { return g ^ ((row >> 1) & 7); }

// Lane l of the 1 KB chunk c of a tile fills LDS slot 64 c + l.
__device__ __forceinline__ uint32_t chunk_off(int chunk, int lane, int64_t ld) {
  const int p = chunk * 64 + lane, row = p >> 3;
  return uint32_t(row) * uint32_t(ld) + uint32_t(slot8(row, p & 7)) * 16u;
}

// The operand of rows r0 + lane % 32 for 64 of the slice's codes: two 16-byte
// reads, lane halves 16 bytes apart in both (any order of k serves, as long as
// both operands have it).
__device__ __forceinline__ i32x8 frag8(const char* t, int r0, int lane, int kk) {
  const int row = r0 + (lane & 31), hh = lane >> 5;
  const u32x4 lo = *reinterpret_cast<const u32x4*>(t + row * kBK + slot8(row, 4 * kk + hh) * 16);
  const u32x4 hi = *reinterpret_cast<const u32x4*>(t + row * kBK + slot8(row, 4 * kk + 2 + hh) * 16);
  return __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One 32 x 32 block of C^T: the lane of half hh holds columns 8 (r / 4) + 4 hh +
// r % 4 of its row.  The halves trade accumulators, so that a lane reads and
// writes eight consecutive columns.
__device__ __forceinline__ void store_block(const Linear8Params& q, f32x16 acc, int64_t m, int n, int hh) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * t + j]),
                                                      __float_as_uint(acc[8 * t + 4 + j]), false, false);
      v[j] = __uint_as_float(s[0]);
      v[4 + j] = __uint_as_float(s[1]);
    }
    const int64_t c = n + 16 * t + 8 * hh;
    if (m < q.M && c < q.N) {
      if (q.r) {
        const bf16x8 rb = *reinterpret_cast<const bf16x8*>(q.r + m * q.ldr + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += float(rb[e]);
      }
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (__bf16)v[e];
      *reinterpret_cast<bf16x8*>(q.out + m * q.ldo + c) = o;
    }
  }
}

template <int ROWS>
constexpr int kScaleBytes = (kScaleSlices * ROWS + 1023) / 1024 * 1024;  // whole wave loads
template <int BM, int BN>
constexpr int kScaleRing = 2 * (kScaleBytes<BM> + kScaleBytes<BN>);

// Scales of the eight slices from `slice` on for ROWS rows from row0 on: [8][ROWS] bytes
// from `lds` on, 1 KB of them by this call's wave.  Rows past the pitch and slices past
// the last one read something or zeros, for rows that are not stored and codes that are zero.
template <int ROWS>
__device__ __forceinline__ void load_scales(uint32_t lds, const Blocks8& b, int64_t row0, int slice, int kblocks,
                                            int part, int lane) {
  const int p = part * 64 + lane, j = p / (ROWS / 16), g = p % (ROWS / 16);
  const int64_t at = slice * b.le + row0, left = kblocks * b.le - at;
  const int64_t most = int64_t(kScaleSlices) * b.le;  // at most 2^31
  const __amdgpu_buffer_rsrc_t r = bytes_rsrc(b.exps + at, left < 0 ? 0 : min(left, min(most, int64_t(0x7fffffff))));
  dma16(lds + uint32_t(part) * 1024u, uint32_t(j) * uint32_t(b.le) + uint32_t(g) * 16u, r);
}

// One BM x BN tile: WM x WN waves, each MB x NB accumulators of 32 x 32; a ring of
// ST slices of both operands, whose loads go out between the products of a step's
// first half.
//
// 25 152 x 7680 x 2560 takes 434-453 us (2.28-2.18 PFLOP/s, by boxes and inputs; the
// library's unscaled product 474), 17 536 x 2560 x 7680 275-286 (2.51-2.41), in loops of
// that call alone.  What it spends there: under counters, in a run of 493 us, the matrix pipes
// are busy 55% of the cycles, at 1.74 GHz.  With one operand row read for all, so that
// every load hits, it takes 337 us where it took 437, with one row written for all 380, with
// both 303 (equal rows also switch fewer bits, so the loads and stores cost at most that).
// A residual's loads go one after another at the tile's end: 4315 x 2560 x 2560
// 31 us without and 34 with one, 25 152 x 2560 x 2560 147 and 185 (25 of them its bytes).
// A form with one wave per SIMD, 128 x 128 accumulators per wave, the next operands
// read between the products and stores left running over the next tile took the same
// 435 (8192 cubed 386-404 against 404-411, but 4315 x 2560 x 2560 36 against 32); loads
// that bring later slices into the L2 early gained nothing, non-temporal stores lost.
template <int MB, int NB, int WM, int WN, int ST>
__device__ __forceinline__ void product8_tile(const Linear8Params& q, char* ring, char* scales, int64_t m0, int n0) {
  constexpr int NW = WM * WN;
  constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
  constexpr int CA = BM / 8 / NW, CW = BN / 8 / NW;
  static_assert(CA * NW * 8 == BM && CW * NW * 8 == BN, "chunks divide over the waves");
  constexpr int kStage = (BM + BN) * kBK, kLoads = CA + CW;
  static_assert(ST * kLoads <= 62, "vmcnt range");
  constexpr int SA = kScaleBytes<BM>, SW = kScaleBytes<BN>;
  static_assert((SA + SW) / 1024 <= NW, "a wave loads at most 1 KB of scales");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int steps = int(blocks8(q.K));

  uint32_t aoff[CA], woff[CW];
#pragma unroll
  for (int i = 0; i < CA; ++i) aoff[i] = chunk_off(i * NW + wave, lane, q.a.ld);
#pragma unroll
  for (int i = 0; i < CW; ++i) woff[i] = chunk_off(i * NW + wave, lane, q.w.ld);
  const int64_t nrec_a = (min(int64_t(BM), q.M - m0) - 1) * q.a.ld + kBK;  // rows past the last load zeros
  const int64_t nrec_w = int64_t(min(BN, q.N - n0) - 1) * q.w.ld + kBK;
  const uint8_t* pa = q.a.codes + m0 * q.a.ld;
  const uint8_t* pw = q.w.codes + n0 * q.w.ld;
  const uint32_t lds0 = lds_u32(ring) + uint32_t(wave) * 1024u;

  const auto issue1 = [&](int slice, uint32_t stage, int l) {
    const bool in = slice < steps;
    const int64_t k0 = in ? int64_t(slice) * kBK : 0;
    if (l < CA) dma16(lds0 + stage + uint32_t(l * NW * 1024), aoff[l], bytes_rsrc(pa + k0, in ? nrec_a : 0));
    else dma16(lds0 + stage + uint32_t(BM * kBK + (l - CA) * NW * 1024), woff[l - CA], bytes_rsrc(pw + k0, in ? nrec_w : 0));
  };
  const auto issue_scales = [&](int slice) {
    const uint32_t at = lds_u32(scales) + uint32_t(slice / kScaleSlices % 2) * (SA + SW);
    if (wave < SA / 1024) load_scales<BM>(at, q.a, m0, slice, steps, wave, lane);
    else if (wave < (SA + SW) / 1024) load_scales<BN>(at + SA, q.w, n0, slice, steps, wave - SA / 1024, lane);
  };

  f32x16 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  issue_scales(0);
#pragma unroll
  for (int s = 0; s < ST - 1; ++s)
#pragma unroll
    for (int l = 0; l < kLoads; ++l) issue1(s, uint32_t(s * kStage), l);
  uint32_t cur = 0, fill = (ST - 1) * kStage;
  for (int s = 0; s < steps; ++s) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 2) * kLoads) : "memory");
    lds_barrier();
    // before the stage's loads: the next step's wait, which counts those, covers these too
    if (s % kScaleSlices == 0) issue_scales(s + kScaleSlices);
    const char* st = ring + cur;
    const char* sc = scales + (s / kScaleSlices % 2) * (SA + SW);
    int ea[MB], ew[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) ea[i] = uint8_t(sc[s % kScaleSlices * BM + wm * 32 * MB + i * 32 + (lane & 31)]);
#pragma unroll
    for (int j = 0; j < NB; ++j) ew[j] = uint8_t(sc[SA + s % kScaleSlices * BN + wn * 32 * NB + j * 32 + (lane & 31)]);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i32x8 fa[MB], fw[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[i] = frag8(st, wm * 32 * MB + i * 32, lane, kk);
#pragma unroll
      for (int j = 0; j < NB; ++j) fw[j] = frag8(st + BM * kBK, wn * 32 * NB + j * 32, lane, kk);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          // C^T block (n rows, m columns): a lane's accumulator is of one output row
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[j], fa[i], acc[i][j], 0, 0, 0, ew[j], 0, ea[i]);
          if (kk == 0) {
            constexpr int NM = MB * NB;
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
              if (l * NM / kLoads == i * NB + j) issue1(s + ST - 1, fill, l);
          }
        }
    }
    cur = cur + kStage == ST * kStage ? 0 : cur + kStage;
    fill = fill + kStage == ST * kStage ? 0 : fill + kStage;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the work-group

#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      store_block(q, acc[i][j], m0 + wm * 32 * MB + i * 32 + (lane & 31), n0 + wn * 32 * NB + j * 32, lane >> 5);
}

template <int MB, int NB, int WM, int WN, int ST>
__global__ __launch_bounds__(WM * WN * 64) void linear8_kernel(const Linear8Params q) {
  constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
  __shared__ __attribute__((aligned(1024))) char ring[ST * (BM + BN) * kBK];
  __shared__ __attribute__((aligned(1024))) char scales[kScaleRing<BM, BN>];
  int64_t row, col;
  grouped_tile<int64_t>(xcd_block(blockIdx.x, gridDim.x), (q.M + BM - 1) / BM, (q.N + BN - 1) / BN, 4, row, col);
  product8_tile<MB, NB, WM, WN, ST>(q, ring, scales, row * BM, int(col * BN));
}

// Few rows, or a small product: reading W is the work, or the launch, and the rows
// are quantised on the way.  A work-group takes 16 MT rows and 32 columns, its
// eight waves a share of the slices each; a wave reads a slice of W and of the rows
// straight into the operands of v_mfma_scale_f32_16x16x128 (lane: row lane % 16, 32
// of the slice's 128 values), the next slice's loads ahead; the four lanes of a row
// agree on the block's maximum, and the waves' sums are added in order through LDS.
// 2 x 7680 x 2560 takes 6.6 us (3 TB/s of W with the launch; 8.1 while each load had
// a branch around it and each value its own conversion); 16 columns per work-group
// up to 4096 of them, which then fit one round: 1 x 2560 x 2560 6.4 -> 4.5 us.
constexpr int kFewWaves = 8;
constexpr int kFewCols = 16 * 256;  // columns up to which 16 per work-group fit one round

template <int MT, int NT, int DEPTH>
__global__ __launch_bounds__(kFewWaves * 64) void linear8_few_kernel(const Linear8Params q) {
  __shared__ f32x4 sums[kFewWaves][MT][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, quarter = lane >> 4;
  const int n0 = int(blockIdx.x) * 16 * NT;
  const int64_t m0 = int64_t(blockIdx.y) * 16 * MT;
  const int steps = int(blocks8(q.K));
  const __amdgpu_buffer_rsrc_t x =
      bytes_rsrc(q.x + m0 * q.ldx, ((min(int64_t(16 * MT), q.M - m0) - 1) * q.ldx + q.K) * 2);
  struct Slice {
    u32x4 w[NT][2], x[MT][4];
    int ew[NT];
  };
  const uint8_t *pw[NT], *pe[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t n = min(n0 + t * 16 + row, q.N - 1);  // columns past the last are not stored
    pw[t] = q.w.codes + n * q.w.ld + quarter * 32;
    pe[t] = q.w.exps + n;
  }
  const auto load = [&](Slice& z, int s) {
    const int64_t k = int64_t(s) * kBK;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      z.w[t][0] = *reinterpret_cast<const u32x4*>(pw[t] + k);
      z.w[t][1] = *reinterpret_cast<const u32x4*>(pw[t] + k + 16);
      z.ew[t] = pe[t][s * q.w.le];
    }
#pragma unroll
    for (int u = 0; u < MT; ++u) {
      const uint32_t c = uint32_t(k) + quarter * 32, at = uint32_t(u * 16 + row) * uint32_t(q.ldx) * 2u + c * 2u;
#pragma unroll
      for (int i = 0; i < 4; ++i) z.x[u][i] = load16(x, at + 16 * i, c + 8 * i < uint32_t(q.K));
    }
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int u = 0; u < MT; ++u)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto add = [&](const Slice& z) {
#pragma unroll
    for (int u = 0; u < MT; ++u) {
      uint32_t a = finite_abs_max(z.x[u]);
      const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
      a = max(r[0], r[1]);
      const auto h = __builtin_amdgcn_permlane32_swap(a, a, false, false);
      a = max(h[0], h[1]);
      const uint32_t byte = exponent_byte(a);
      u32x8 fx;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 c = codes8(z.x[u][i], byte);
        fx[2 * i] = c[0];
        fx[2 * i + 1] = c[1];
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const u32x8 fw = __builtin_shufflevector(z.w[t][0], z.w[t][1], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[u][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            __builtin_bit_cast(i32x8, fw), __builtin_bit_cast(i32x8, fx), acc[u][t], 0, 0, 0, z.ew[t], 0, int(byte));
      }
    }
  };
  Slice z[DEPTH];
  int s = wave;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (s + d * kFewWaves < steps) load(z[d], s + d * kFewWaves);
  while (s < steps) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d, s += kFewWaves) {
      if (s < steps) add(z[d]);
      if (s + DEPTH * kFewWaves < steps) load(z[d], s + DEPTH * kFewWaves);
    }
  }
#pragma unroll
  for (int u = 0; u < MT; ++u)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][u][t][lane] = acc[u][t];
  __syncthreads();
  for (int i = wave; i < MT * NT; i += kFewWaves) {
    const int u = i / NT, t = i % NT;
    f32x4 v = sums[0][u][t][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) v += sums[w][u][t][lane];
    const int64_t m = m0 + u * 16 + row;
    const int n = n0 + t * 16 + quarter * 4;  // the accumulator of 16 x 16: column lane % 16, rows 4 (lane / 16) ..
    if (m >= q.M || n >= q.N) continue;
    if (q.r) {
      const bf16x4 rb = *reinterpret_cast<const bf16x4*>(q.r + m * q.ldr + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += float(rb[e]);
    }
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)v[e];
    *reinterpret_cast<bf16x4*>(q.out + m * q.ldo + n) = o;
  }
}

template <int MB, int NB, int WM, int WN, int ST>
void launch_tile(const Linear8Params& q, hipStream_t s) {
  constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
  hipLaunchKernelGGL((linear8_kernel<MB, NB, WM, WN, ST>), dim3((q.M + BM - 1) / BM * ((q.N + BN - 1) / BN)),
                     dim3(WM * WN * 64), 0, s, q);
}

}  // namespace

int launch_linear8(const Linear8Params& q, int32_t tile, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (tile) {
    case 0: launch_tile<4, 2, 2, 4, 2>(q, s); break;
    case 1: launch_tile<3, 2, 2, 4, 2>(q, s); break;
    case 2: launch_tile<2, 2, 4, 2, 3>(q, s); break;
    case 3: launch_tile<2, 2, 2, 2, 4>(q, s); break;
    case 4: launch_tile<2, 1, 1, 4, 6>(q, s); break;
    default: launch_tile<1, 1, 2, 2, 8>(q, s); break;
  }
  return int(hipGetLastError());
}

int launch_linear8_few(const Linear8Params& q, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto launch = [&](auto kernel, int rows, int cols) {
    hipLaunchKernelGGL(kernel, dim3((q.N + cols - 1) / cols, (q.M + rows - 1) / rows), dim3(kFewWaves * 64), 0, s, q);
  };
  if (q.M > 16) launch(linear8_few_kernel<2, 2, 2>, 32, 32);
  else if (q.N > kFewCols) launch(linear8_few_kernel<1, 2, 3>, 16, 32);
  else launch(linear8_few_kernel<1, 1, 4>, 16, 16);
  return int(hipGetLastError());
}

}  // namespace rc
