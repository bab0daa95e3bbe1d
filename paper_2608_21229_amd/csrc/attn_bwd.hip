// Gradient of block-masked attention for gfx950.
//
// With p_ij = exp(scale q_i k_j - lse_i) over the visible pairs and D_i =
// sum_d dO_id O_id - dlse_i:
//   ds_ij = p_ij (dO_i v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j   dk_j = scale sum_i ds_ij q_i   dv_j = sum_i p_ij dO_i
//
// Five products per pair (S = QK, dP = dO V, dV, dK, dQ).  dV and dK sum over
// queries, dQ over keys, so one pass over the pairs would have to add one of
// them to memory from many work-groups: in an order that changes the sums, or
// through one fp32 partial of dQ per 256 keys (two 1024-pixel samples of 24
// heads: 7 GB written and read, 3 ms).  Two kinds of work-groups in one launch
// compute seven products instead and write every output once: those that hold
// 256 (128) keys stream the queries that see them (S, dP, dV, dK), those that hold
// 256 (128) queries stream the keys they see (S, dP, dQ).
//
// Layout of the work.  A wave holds 64 own rows as two blocks of 32 (operands in
// registers, sums in accumulation registers), so that a fragment read from LDS
// feeds two products (one block and eight waves: 817 us for the ragged D = 64
// case against 644).  Few rows or heads take one block per wave and own tiles of
// 128 rows on twice the work-groups, each tile in two thirds of the time (343 rows,
// one head: 21.5 -> 15.8 us; but 22 heads of 1516 rows: 95.5 -> 103.8, so the planner
// weighs both).  Four waves share a 3-stage ring of 64 streamed rows of two tensors,
// loaded straight to LDS (4 to 6 stages measured the same).  One wave per SIMD, so
// nothing but its own order hides latency: the loop is one stream of slots, each a
// product followed by its share of the other work (a fragment read PF products
// ahead, one or two exponentials, a pair of ds, a load of the next stage), and
// fences keep the compiler from moving work between slots.  The scores of the next
// 32 rows are computed before dK (dQ) of the present ones, so that their
// exponentials have products to hide behind.
//
// Rounding: P and ds are rounded to bf16 (off by at most 2^-8 of each) as operands
// of the products dV, dK and dQ; scores, exponentials, dP and all sums stay fp32.
// The statistics enter in fp32: keys start S from -lse / scale and dP from -D (a
// row's value is the accumulator's first addend), queries subtract them.
//
// What bounds it (two 1024-pixel samples, 24 heads, D = 128): 3.66 ms (to 3.84 on other
// machines; 4.0 in a process's first calls, whose clock is lower), 967 TFLOP/s
// of five products, 1350 of the seven computed, which is what a large library
// matrix product reaches here; the matrix pipes are busy 71% of the cycles and the
// clock falls to 1.7 GHz.  With exponentials, ds, fragment reads and loads taken out
// the same products take 2.83 ms; the loads alone are 2%, the reads 3%.
// D = 64 has half the products per exponential and is bound by issue: 613 us for the
// ragged case, 501 without exponentials and ds.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_layer.h"

namespace rc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) const bf16x8 lds_cbf16x8;
typedef __attribute__((address_space(3))) const f32x4 lds_cf32x4;

constexpr int kTile = 64;  // streamed rows per tile

__device__ __forceinline__ uint32_t lds_u32(const char* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_void*)p));
}
__device__ __forceinline__ void dma16(uint32_t lds, uint32_t voff, __amdgpu_buffer_rsrc_t rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4(uint32_t lds, uint32_t voff, __amdgpu_buffer_rsrc_t rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// The lane index, computed where it is used: kept, it would be one more
// register across the loop.
__device__ __forceinline__ uint32_t fresh_lane() {
  uint32_t l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// A wave-uniform 64-bit product, which the compiler computes with vector
// instructions, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(x));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(uint64_t(x) >> 32));
  return int64_t(uint64_t(hi) << 32 | lo);
}

// D: head width; KV: own rows are keys; NB blocks of 32 own rows per wave; NW
// waves; ST stages.
template <int D, bool KV, int NB, int NW, int ST>
struct Bwd {
  static constexpr int GR = D / 8, DC = D / 16, DB = D / 32;
  static constexpr int kT = kTile * D * 2;         // bytes of one streamed tile of one tensor
  static constexpr int kStage = 2 * kT + 1024;     // both tensors, then -lse/scale and -D of the rows
  static constexpr int kLoads = 2 * kT / 1024 / NW + 1;
  static constexpr int kOwn = 32 * NB * NW;
};

// 16-byte granule g of row r lies at slot g ^ swz(r).  16 consecutive rows at
// one granule (128-bit reads) and 4 consecutive rows at 4 consecutive granules
// (transpose reads) hit 16 distinct bank groups; a 128-byte row fills half of
// the banks, so there bit 0 of the row already tells two halves apart.
template <int D>
__device__ __forceinline__ int swz(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return ((row & 2) << 1) | ((row >> 1) & 2) | ((row >> 3) & 1);
}

// One 32 x 32 block of an output: the lane of half hh holds columns 8 (r / 4) + 4
// hh + r % 4 of its row.  The halves trade registers, so that a lane owns eight
// consecutive columns of each 16 and stores 16 bytes.
__device__ __forceinline__ void store_block(uint16_t* out, const f32x16& acc, float f, bool in) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * i + e] * f),
                                                      __float_as_uint(acc[8 * i + 4 + e] * f), false, false);
      o[e] = (__bf16)__uint_as_float(x[0]);
      o[4 + e] = (__bf16)__uint_as_float(x[1]);
    }
    if (in) *reinterpret_cast<bf16x8*>(out + 16 * i) = o;
  }
}

// One piece of an own tile: its share of the streamed rows, and the stores.
//
// The accumulator products are single statements of assembly ("+a"): the
// compiler would move the sums of 16 registers between files around every
// product.  It does not see their hazards: two wait states lie between a vector
// instruction and a product that reads its result (a read, a fence's slot), and
// `settle` waits for the last ones; both are checked in the built assembly by a
// test.
template <int D, bool KV, int NB, int NW, int ST>
__device__ __forceinline__ void bwd_tile(const BwdParams& p, char* ring, const BwdSeg seg, int bh, int t, int piece) {
  using T = Bwd<D, KV, NB, NW, ST>;
  // fragments read ahead of their MFMAs (two blocks at D = 128 have no registers for a third)
  constexpr int PF = NB == 1 ? 4 : D == 64 ? 3 : 2;
  constexpr int GR = T::GR, DC = T::DC, DB = T::DB, kT = T::kT;
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = __builtin_amdgcn_readfirstlane(bh / p.H), h = bh - b * p.H;
  const int own0 = t * T::kOwn + wave * 32 * NB;  // inside the segment

  const int64_t o_st = int64_t(p.H) * D;
  const int64_t q_base = uniform(int64_t(b) * p.n_rows * p.st + int64_t(h) * D);
  const int64_t o_base = uniform(int64_t(b) * p.n_rows * o_st + int64_t(h) * D);
  const int64_t s_base = uniform(int64_t(bh) * p.n_rows);
  const uint16_t* x1 = (KV ? p.k : p.q) + q_base;
  const uint16_t* x2 = KV ? p.v + q_base : p.d_o + o_base;
  const int64_t x2_st = KV ? p.st : o_st;
  const uint16_t* y1 = (KV ? p.q : p.k) + q_base;
  const uint16_t* y2 = KV ? p.d_o + o_base : p.v + q_base;
  const int64_t y1_st = p.st, y2_st = KV ? o_st : p.st;

  // own operands: row lane % 32, d = 16 c + 8 hh .. +7
  bf16x8 f1[NB][DC], f2[NB][DC];
  float cs[NB], cd[NB];  // dQ: -lse log2(e) and -D of the lane's query
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = own0 + nb * 32 + (lane & 31);
    const bool in = r < seg.len;
    const int64_t row = seg.row0 + (in ? r : 0);
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      bf16x8 a = *reinterpret_cast<const bf16x8*>(x1 + row * p.st + c * 16 + hh * 8);
      bf16x8 e = *reinterpret_cast<const bf16x8*>(x2 + row * x2_st + c * 16 + hh * 8);
      if (!in) a = e = bf16x8{};
      f1[nb][c] = a;
      f2[nb][c] = e;
    }
    if constexpr (!KV) {
      cs[nb] = in ? p.nlse[s_base + row] * p.scale_log2 : 0.f;
      cd[nb] = in ? p.ndelta[s_base + row] : 0.f;
    }
  }

  f32x16 acc1[NB][DB], acc2[KV ? NB : 1][DB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        acc1[nb][d][i] = 0.f;
        if constexpr (KV) acc2[nb][d][i] = 0.f;
      }

  // Streamed tiles.  The loading cursor keeps its range in scalar registers; the
  // range table is read again only at a range's end.
  int n_tiles = 0;
  for (int i = 0; i < seg.nr; ++i) n_tiles += (p.range[seg.r0 + i].len + kTile - 1) / kTile;
  int skip = int(int64_t(n_tiles) * piece / seg.splits);  // tiles of the pieces before
  n_tiles = int(int64_t(n_tiles) * (piece + 1) / seg.splits) - skip;
  int ir = seg.r0, rem = 0;
  for (; ir + 1 < seg.r0 + seg.nr; ++ir) {
    const int n = (p.range[ir].len + kTile - 1) / kTile;
    if (skip < n) break;
    skip -= n;
  }
  int left = n_tiles;  // tiles to load
  const uint16_t *l1 = y1, *l2 = y2;
  const float* ls = ((wave & 1) ? p.ndelta : p.nlse) + s_base;
  const auto load_range = [&](int tile) {
    const BwdRange rg = p.range[ir];
    const int64_t row = rg.start + int64_t(tile) * kTile;
    l1 = y1 + uniform(row * y1_st);
    l2 = y2 + uniform(row * y2_st);
    ls = ((wave & 1) ? p.ndelta : p.nlse) + s_base + row;
    rem = rg.len - tile * kTile;
  };
  const auto advance = [&] {
    rem -= kTile;
    if (--left <= 0) {  // past the piece: the ring's last loads bring zeros
      rem = 0;
    } else if (rem > 0) {
      l1 += kTile * y1_st;
      l2 += kTile * y2_st;
      ls += kTile;
    } else {
      ++ir;
      load_range(0);
    }
  };
  if (n_tiles > 0) load_range(skip);
  const uint32_t lds0 = lds_u32(ring) + wave * 1024;
  // a lane's byte offsets in the tiles of Y1 and Y2, computed where a tile is loaded (fresh_lane)
  uint32_t voff1 = 0, voff2 = 0;
  const auto lane_offsets = [&] {
    const int l = int(fresh_lane()), row = wave * (512 / D) + l / GR;
    const uint32_t gran = uint32_t((l % GR) ^ swz<D>(row)) * 16;
    voff1 = uint32_t(row) * uint32_t(y1_st * 2) + gran;
    voff2 = uint32_t(row) * uint32_t(y2_st * 2) + gran;
  };
  // a wave's chunks lie a multiple of 16 rows apart, so their lane offsets are the same
  constexpr int CH = kT / 1024 / NW, kStep = 1024 * NW / (D * 2);
  static_assert(kStep % 16 == 0, "one swizzle for a wave's chunks");
  constexpr int kLoads = 2 * CH + (KV ? 1 : 0);
  // Load l of the cursor's tile; rows past the range lie beyond the record
  // count and arrive as zeros.
  const uint32_t step1 = uint32_t(y1_st * 2) * kStep, step2 = uint32_t(y2_st * 2) * kStep;
  __amdgpu_buffer_rsrc_t rs1, rs2, rsl;
  const auto rsrc = [](const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, __builtin_bit_cast(int, bytes),
                                             0x00020000);
  };
  const auto start_tile = [&] {
    const uint32_t n = min(kTile, rem);
    rs1 = rsrc(l1, n * uint32_t(y1_st * 2));
    rs2 = rsrc(l2, n * uint32_t(y2_st * 2));
    if constexpr (KV) rsl = rsrc(ls, n * 4);
  };
  const auto issue1 = [&](uint32_t stage, int l) {
    const int i = l / 2;
    if (l >= 2 * CH) dma4(lds_u32(ring) + stage + 2 * kT + (wave & 1) * 256, fresh_lane() * 4, rsl);
    else if (l & 1) dma16(lds0 + stage + kT + i * NW * 1024, voff2 + i * step2, rs2);
    else dma16(lds0 + stage + i * NW * 1024, voff1 + i * step1, rs1);
  };
  const auto issue = [&](uint32_t stage) {
    start_tile();
    lane_offsets();
#pragma unroll
    for (int l = 0; l < kLoads; ++l) issue1(stage, l);
  };
  int valid[ST];  // rows of the tile computed and of those loaded after it
#pragma unroll
  for (int s = 0; s < ST - 1; ++s) {
    valid[s] = min(kTile, rem);
    issue(s * T::kStage);
    advance();
  }

  // Fragment addresses (LDS bytes): rows lane % 32 of a sub-block, granule
  // hh; the two transpose reads, rows 4 hh + li / 4 and 8 further.  Granule 2 c
  // + hh and d block d are the base XOR a constant, since a stage starts at a
  // multiple of 1 KB.
  const int li = lane & 15;
  uint32_t kc = lds_u32(ring) + (lane & 31) * D * 2 + 16 * (swz<D>(lane & 31) ^ hh);
  const int gc = 2 * ((lane >> 4) & 1) + ((li & 3) >> 1);
  const int r0 = 4 * hh + (li >> 2);
  uint32_t t0 = lds_u32(ring) + r0 * D * 2 + 16 * (gc ^ swz<D>(r0)) + 8 * (li & 1);
  constexpr uint32_t k8 = 16 * (D == 128 ? 2 : 1);  // 8 rows further the slot differs in this bit
  const auto rd = [](uint32_t base, int c, int off) {
    return *reinterpret_cast<lds_cbf16x8*>((base ^ uint32_t(32 * c)) + uint32_t(off));
  };
  const auto tr = [](uint32_t base, int f, int off) {
    const int ks = f / DB, d = f % DB;
    const uint32_t at = uint32_t(off + ks * 16 * D * 2);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)((base ^ uint32_t(64 * d)) + at));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)((base ^ uint32_t(64 * d) ^ k8) + at + 8 * D * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const auto rows16 = [&](uint32_t stage, int off) {  // a statistic of a sub-block's 32 rows, in accumulator order
    const uint32_t base = lds_u32(ring) + stage + (fresh_lane() >> 5) * 16;
    off += 2 * kT;
    f32x16 l;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = *reinterpret_cast<lds_cf32x4*>(base + uint32_t(off + g * 32));
#pragma unroll
      for (int e = 0; e < 4; ++e) l[4 * g + e] = x[e];
    }
    return l;
  };
  f32x16 s[NB], dp[NB];
  f32x16 nl{}, nd{};  // dK, dV: the rows' -lse/scale and -D, the products' first addends, read ahead
  // dQ: a lane's -D is one value.  At D = 64 there are registers for it as dP's first addend
  // (623 -> 613 us for the ragged case), at D = 128 it is added.
  constexpr bool kAdd = !KV && D == 128;
  f32x16 od[KV || kAdd ? 1 : NB];
  if constexpr (!KV && !kAdd) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) od[nb][r] = cd[nb];
      asm volatile("" : "+v"(od[nb]));
    }
  }
  const auto start = [](f32x16 (&x)[NB], const f32x16& c) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[nb][r] = KV ? c[r] : 0.f;
  };
  const auto mm = [](bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); };
  const auto am = [](bf16x8 a, bf16x8 b, f32x16& c) {
    asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  };
  // Score e = 0 .. 16 NB - 1 of the lane: the accumulators' first halves of the
  // blocks, then the second ones.  The argument of a score is computed kAhead
  // scores before its exponential.  (An empty statement that pins a value to
  // its place counts as its producer: the compiler puts a wait state between it
  // and a use right behind it.)
  constexpr int kAhead = D == 64 || NB == 1 ? 2 : 1;
  float arg[kAhead];
  constexpr int NU = 16 * NB;
  const auto make_arg = [&](int e) {
    const int nb = (e >> 3) % NB;
    const float x = s[nb][8 * (e / (8 * NB)) + (e & 7)];
    float& a = arg[e % kAhead];
    a = KV ? x * p.scale_log2 : __builtin_fmaf(x, p.scale_log2, cs[nb]);
    asm volatile("" : "+v"(a));
  };
  const auto first_args = [&] {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) make_arg(e);
  };
  const auto unit = [&](int e) {
    float t = __builtin_amdgcn_exp2f(arg[e % kAhead]);
    if (e + kAhead < NU) make_arg(e + kAhead);
    asm volatile("" : "+v"(t));  // stays in its slot
    s[(e >> 3) % NB][8 * (e / (8 * NB)) + (e & 7)] = t;
  };
  const auto units = [&](int from, int to, int slot, int slots) {
#pragma unroll
    for (int e = 0; e < NU; ++e)
      if (e >= from && e < to && (e - from) * slots / (to - from) == slot) unit(e);
  };
  // dQ: scores of keys past the range are -inf (p = 0).  dK, dV need no mask:
  // rows past the range are zeros with zero statistics, so ds = 0 and dO = 0.
  const auto mask = [&](int valid) {
    if (KV || valid >= 32) return;
    const int lim = valid - 4 * hh;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= lim) s[nb][r] = -INFINITY;
  };
  // Exponentials of a sub-block: kE1 beside dK (dQ) of the one before, up to
  // kE2 beside its dP, the rest beside the first half of its dV.
  constexpr int kE1 = NU * (KV ? 11 : 16) / 32, kE2 = NU * (KV ? 24 : 32) / 32;
  constexpr int R = PF + 1;
  bf16x8 fr[R];
  uint32_t cur = 0, nxt = T::kStage, fill = (ST - 1) * T::kStage;
  if (n_tiles > 0) {  // S(0) and its first exponentials
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 2) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    if constexpr (KV) {
      nl = rows16(0, 0);
      nd = rows16(0, 256);
    }
    start(s, nl);
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      const bf16x8 a = rd(kc, c, 0);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[nb] = mm(a, f1[nb][c], s[nb]);
    }
    mask(valid[0]);
    first_args();
#pragma unroll
    for (int e = 0; e < kE1; ++e) unit(e);
#pragma unroll
    for (int g = 0; g < PF; ++g) fr[g] = rd(kc, g, kT);
  }
  for (int tile = 0; tile < n_tiles; ++tile) {
    const uint32_t step = nxt - cur;  // to the next stage
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // at D = 128 the registers are full: addresses are recomputed (one XOR a read), not kept
      if constexpr (D == 128) asm volatile("" : "+v"(kc), "+v"(t0));
      const uint32_t kn = j == 0 ? kc : kc + step;      // the next sub-block: rows, statistics
      const uint32_t sn = j == 0 ? cur : nxt;
      constexpr int kSub = 32 * D * 2;
      const int here = j * kSub, there = j == 0 ? kSub : 0, sthere = j == 0 ? 128 : 0;
      constexpr int GV = KV ? 2 * DB : 0;               // fragments of dV
      constexpr int G = DC + GV + DC + 2 * DB;          // of the sub-block
      const auto read = [&](int g) {
        if (g < DC) return rd(kc, g, kT + here);
        if (g < DC + GV) return tr(t0, g - DC, kT + here);
        if (g < DC + GV + DC) return rd(kn, g - DC - GV, there);
        if (g < G) return tr(t0, g - DC - GV - DC, here);
        return rd(kn, g - G, kT + there);
      };
      bf16x8 pf[NB][2], df[NB][2];
      const auto pack = [&](int ks, int nb) {
#pragma unroll
        for (int r = 0; r < 8; ++r) pf[nb][ks][r] = (__bf16)s[nb][8 * ks + r];
        asm volatile("" : "+v"(pf[nb][ks]));
      };
      // Pairs of ds = p dP.  A pair's dP is pinned kAhead pairs before its use, so that it
      // is not computed in an earlier slot and other instructions lie in between.
      float dx[kAhead][2];
      const auto pin_pair = [&](int e) {
        const int ks = e / (4 * NB), nb = (e >> 2) % NB, r = 2 * (e & 3);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          dx[e % kAhead][i] = dp[nb][8 * ks + r + i];
          asm volatile("" : "+v"(dx[e % kAhead][i]));
        }
      };
      const auto first_pairs = [&] {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) pin_pair(e);
      };
      const auto ds = [&](int from, int to, int slot, int slots) {
#pragma unroll
        for (int e = 0; e < NU / 2; ++e)
          if (e >= from && e < to && (e - from) * slots / (to - from) == slot) {
            const int ks = e / (4 * NB), nb = (e >> 2) % NB, r = 2 * (e & 3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float x = dx[e % kAhead][i];
              df[nb][ks][r + i] = (__bf16)(s[nb][8 * ks + r + i] * (kAdd ? x + cd[nb] : x));
            }
            asm volatile("" : "+v"(df[nb][ks]));
            if (e + kAhead < NU / 2) pin_pair(e + kAhead);
          }
      };
      const auto next_tile = [&] {  // the next tile has landed everywhere, its stage's last readers are done
        if (j == 0) return;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 3) * kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        start_tile();
      };
      if constexpr (KV || kAdd) start(dp, nd);
      else
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) dp[nb] = od[nb];
      fence();
      int g = 0;
      // dP(i)
#pragma unroll
      for (int c = 0; c < DC; ++c, ++g) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          dp[nb] = mm(fr[g % R], f2[nb][c], dp[nb]);
          fence();
          if (!KV && nb == 0 && g + PF == DC) next_tile();  // before the first read of S(i + 1)'s rows
          if (nb == 0) fr[(g + PF) % R] = read(g + PF);
          units(kE1, kE2, NB * c + nb, NB * DC);
          if (KV && nb == 0 && c >= DC - 2 && c - (DC - 2) < NB) pack(0, c - (DC - 2));
          fence();
        }
      }
      if constexpr (KV) {
        next_tile();  // S(i + 1)'s rows are read from dV on
        fence();
        // dV(i)
#pragma unroll
        for (int f = 0; f < 2 * DB; ++f, ++g) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            am(fr[g % R], pf[nb][f / DB], acc2[nb][f % DB]);
            fence();
            if (nb == 0) fr[(g + PF) % R] = read(g + PF);
            if (f < DB) units(kE2, NU, NB * f + nb, NB * DB);
            else ds(0, NU / 4, NB * (f - DB) + nb, NB * DB);
            if (f == DB - 1) pack(1, nb);
            if (f == DB - 1 && nb == NB - 1) first_pairs();
            if (f == DB - 1 && NB == 1) asm volatile("s_nop 1");  // the next product reads what was just packed
            if (f == 2 * DB - 1 && nb == 0) nl = rows16(sn, sthere);
            fence();
          }
        }
      }
      // S(i + 1)
      f32x16 s2[NB];
      start(s2, nl);
#pragma unroll
      for (int c = 0; c < DC; ++c, ++g) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          s2[nb] = mm(fr[g % R], f1[nb][c], s2[nb]);
          fence();
          if (nb == 0) fr[(g + PF) % R] = read(g + PF);
          if (KV) ds(NU / 4, NU / 2, NB * c + nb, NB * DC / 2);
          else ds(0, NU / 2, NB * c + nb - 2, NB * DC - 2);
          if (!KV && c == 0 && nb == NB - 1) first_pairs();
          fence();
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[nb] = s2[nb];
      if (j == 1) {
        valid[ST - 1] = min(kTile, rem);
#pragma unroll
        for (int s = 0; s < ST - 1; ++s) valid[s] = valid[s + 1];
      }
      mask(j == 0 ? valid[0] - 32 : valid[0]);
      fence();
      // dK(i) or dQ(i)
#pragma unroll
      for (int f = 0; f < 2 * DB; ++f, ++g) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          am(fr[g % R], df[nb][f / DB], acc1[nb][f % DB]);
          fence();
          if (nb == 0) fr[(g + PF) % R] = read(g + PF);
          if (KV && f == 2 * DB - 2 && nb == 0) nd = rows16(sn, sthere + 256);
          if (NB * f + nb == 1) first_args();
          units(0, kE1, NB * f + nb - 2, 2 * NB * DB - 2);
          if (j == 1)
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
              if (l * (2 * NB * DB) / kLoads == NB * f + nb) issue1(fill, l);
          fence();
        }
      }
      bf16x8 first[PF];  // the next sub-block's first fragments
#pragma unroll
      for (int i = 0; i < PF; ++i) first[i] = fr[(G + i) % R];
#pragma unroll
      for (int i = 0; i < PF; ++i) fr[i] = first[i];
    }
    advance();
    kc += step;
    t0 += step;
    cur = nxt;
    nxt = nxt + T::kStage == ST * T::kStage ? 0 : nxt + T::kStage;
    fill = fill + T::kStage == ST * T::kStage ? 0 : fill + T::kStage;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the work-group

  // The compiler does not see that the accumulators come from MFMAs: the last
  // of them are waited for here, before the first read.
  const auto settle = [](f32x16& c) { asm volatile("s_nop 15\n\ts_nop 3" : "+a"(c)); };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      settle(acc1[nb][d]);
      if constexpr (KV) settle(acc2[nb][d]);
    }

  const int lane_ = int(fresh_lane());
  if (seg.splits > 1) {  // a partial: 1 KB runs, in accumulator order
    const int own_tiles = (seg.len + T::kOwn - 1) / T::kOwn;
    const int64_t slot = int64_t(p.B) * p.H * seg.slot0 +
                         ((int64_t(bh) * own_tiles + t) * seg.splits + piece) * (KV ? 2 : 1);
    f32x4* out = reinterpret_cast<f32x4*>(p.partial + slot * T::kOwn * D) + lane_;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = (((wave * NB + nb) * DB + d) * 4 + i) * 64;
          const f32x16& a = acc1[nb][d];
          out[at] = f32x4{a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3]};
          if constexpr (KV) {
            const f32x16& c = acc2[nb][d];
            out[at + T::kOwn * D / 4] = f32x4{c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]};
          }
        }
    return;
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = own0 + nb * 32 + (lane_ & 31);
    const int64_t at = (int64_t(b) * p.n_rows + seg.row0 + r) * p.g_st + int64_t(h) * D + 8 * (lane_ >> 5);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      store_block((KV ? p.dk : p.dq) + at + d * 32, acc1[nb][d], p.scale, r < seg.len);
      if constexpr (KV) store_block(p.dv + at + d * 32, acc2[nb][d], 1.f, r < seg.len);
    }
  }
}

template <int D, int NB, int NW, int ST>
__global__ __launch_bounds__(64 * NW, NW / 4) void attn_bwd_kernel(const BwdParams p) {
  __shared__ __attribute__((aligned(1024))) char ring[ST * Bwd<D, true, NB, NW, ST>::kStage];
  // The hardware deals work-groups round-robin to the 8 XCDs.  Where the heads
  // divide over them, an XCD takes whole heads, whose streamed rows then share
  // its L2 (two 1024-pixel samples of 24 heads: 4.10 ms, and 4.19 without).
  // Work-groups run in order of their segment (longest first), then batch and
  // head, then tile.
  const int bhs = p.B * p.H;
  const bool split = bhs % 8 == 0;
  const int hx = split ? bhs / 8 : bhs;
  const int w = split ? blockIdx.x >> 3 : blockIdx.x;
  int si = 0;
  while (si + 1 < p.n_seg && p.seg[si + 1].piece0 * hx <= w) ++si;
  const BwdSeg seg = p.seg[si];
  constexpr int kOwn = Bwd<D, true, NB, NW, ST>::kOwn;
  const int in_seg = w - seg.piece0 * hx, pieces = (seg.len + kOwn - 1) / kOwn * seg.splits;
  // (quotients come from vector instructions; as scalars they take no registers across the loops)
  const int head = __builtin_amdgcn_readfirstlane(in_seg / pieces), in_head = in_seg - head * pieces;
  const int t = __builtin_amdgcn_readfirstlane(in_head / seg.splits), piece = in_head - t * seg.splits;
  const int bh = (split ? (blockIdx.x & 7) * hx : 0) + head;
  if (seg.keys) bwd_tile<D, true, NB, NW, ST>(p, ring, seg, bh, t, piece);
  else bwd_tile<D, false, NB, NW, ST>(p, ring, seg, bh, t, piece);
}

// The pieces of split tiles, summed in order (fp32), bound by the partials' bytes.
// With few heads the split pays for it: five references, one head 897 us unsplit,
// 335 split; a 512-pixel edit, three heads 142 and 64.  A wave takes one 32 x 32 block; its
// partials' loads are in flight together, four pieces at a time.
template <int D, int kOwn>
__global__ __launch_bounds__(256) void attn_bwd_merge_kernel(const BwdParams p) {
  constexpr int DB = D / 32, kBlocks = kOwn / 32 * DB;  // blocks of one output of a tile
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  int64_t w = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t bhs = int64_t(p.B) * p.H;
  int si = 0;
  int64_t own = 0;
  for (; si < p.n_seg; ++si) {
    if (p.seg[si].splits <= 1) continue;
    own = (p.seg[si].len + kOwn - 1) / kOwn;
    const int64_t n = bhs * own * (1 + p.seg[si].keys) * kBlocks;
    if (w < n) break;
    w -= n;
  }
  if (si == p.n_seg) return;
  const BwdSeg seg = p.seg[si];
  const int outs = 1 + seg.keys;
  const int block = int(w % kBlocks), out = int(w / kBlocks % outs);
  const int64_t tile = w / kBlocks / outs;  // (batch, head), own tile
  const f32x4* src = reinterpret_cast<const f32x4*>(p.partial + (bhs * seg.slot0 + tile * seg.splits * outs + out) * kOwn * D) +
                     block * 256 + lane;
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int s0 = 0; s0 < seg.splits; s0 += 4) {
    f32x4 v[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[j][i] = s0 + j < seg.splits ? src[int64_t(s0 + j) * outs * kOwn * D / 4 + i * 64] : f32x4{};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] += v[j][r / 4][r % 4];
  }
  const int64_t bh = tile / own;
  const int r = int(tile % own) * kOwn + block / DB * 32 + (lane & 31);
  uint16_t* dst = seg.keys ? (out ? p.dv : p.dk) : p.dq;
  dst += ((bh / p.H) * p.n_rows + seg.row0 + r) * p.g_st + (bh % p.H) * D + block % DB * 32 + 8 * hh;
  store_block(dst, acc, seg.keys && out ? 1.f : p.scale, r < seg.len);
}

// -lse / scale and -D of every row; rows that read nothing get -inf and 0.  One
// pass over o and d_o, 16 bytes a lane: HBM-bound (47 us for the 215 MB of two 1024-pixel samples).
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_rows_kernel(const BwdParams p) {
  constexpr int L = D / 8;
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) / L;  // (b, n, h)
  const int g = threadIdx.x % L;
  if (i >= int64_t(p.B) * p.n_rows * p.H) return;
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p.o + i * D + g * 8);
  const bf16x8 c = *reinterpret_cast<const bf16x8*>(p.d_o + i * D + g * 8);
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += float(a[e]) * float(c[e]);
#pragma unroll
  for (int m = L / 2; m > 0; m >>= 1) s += __shfl_xor(s, m);
  if (g != 0) return;
  const int h = int(i % p.H);
  const int64_t bn = i / p.H, b = bn / p.n_rows, n = bn % p.n_rows;
  const int64_t at = (b * p.H + h) * p.n_rows + n;
  const float l = p.lse[at];
  const bool none = l == -INFINITY;
  p.nlse[at] = none ? -INFINITY : -l / p.scale;
  p.ndelta[at] = none ? 0.f : (p.dlse ? p.dlse[at] : 0.f) - s;
}

template <int D, int NB>
void launch(const BwdParams& p, hipStream_t s) {
  constexpr int NW = 4, ST = 3, kOwn = 32 * NB * NW;
  const int64_t rows = int64_t(p.B) * p.n_rows * p.H;
  hipLaunchKernelGGL(attn_bwd_rows_kernel<D>, dim3((rows * (D / 8) + 255) / 256), dim3(256), 0, s, p);
  const int64_t bh = int64_t(p.B) * p.H;
  hipLaunchKernelGGL((attn_bwd_kernel<D, NB, NW, ST>), dim3(bh * p.n_pieces), dim3(64 * NW), 0, s, p);
  int64_t tiles = 0;
  for (int i = 0; i < p.n_seg; ++i)
    if (p.seg[i].splits > 1) tiles += (p.seg[i].len + kOwn - 1) / kOwn * (1 + p.seg[i].keys);
  if (tiles > 0)  // four blocks of 32 x 32 per work-group
    hipLaunchKernelGGL((attn_bwd_merge_kernel<D, kOwn>), dim3(bh * tiles * (kOwn * D / 4096)), dim3(256), 0, s, p);
}

}  // namespace

int launch_attention_bwd(const BwdParams& p, int D, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.own == 128) D == 64 ? launch<64, 1>(p, s) : launch<128, 1>(p, s);
  else D == 64 ? launch<64, 2>(p, s) : launch<128, 2>(p, s);
  return int(hipGetLastError());
}

}  // namespace rc
