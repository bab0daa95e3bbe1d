// Gradient of block-masked attention for gfx950.
//
// With p_ij = exp(scale q_i k_j - lse_i) over the visible pairs and D_i =
// sum_d dO_id O_id - dlse_i:
//   ds_ij = p_ij (dO_i v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j   dk_j = scale sum_i ds_ij q_i   dv_j = sum_i p_ij dO_i
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

template <int D, bool KV, int NB, int NW, int ST>
struct Bwd {
  static constexpr int GR = D / 8, DC = D / 16, DB = D / 32;
  static constexpr int kT = kTile * D * 2;         // bytes of one streamed tile of one tensor
  static constexpr int kStage = 2 * kT + 1024;     // both tensors, then -lse/scale and -D of the rows
  static constexpr int kLoads = 2 * kT / 1024 / NW + 1;
  static constexpr int kOwn = 32 * NB * NW;
};

__device__ __forceinline__ int swz(int row, int gr) { return (((row & 3) << 2) | ((row >> 2) & 3)) & (gr - 1); }

template <int D, bool KV, int NB, int NW, int ST>
__global__ __launch_bounds__(64 * NW, NW / 4) void attn_bwd_kernel(const BwdParams p) {
  using T = Bwd<D, KV, NB, NW, ST>;
  constexpr int GR = T::GR, DC = T::DC, DB = T::DB, kT = T::kT;
  __shared__ __attribute__((aligned(1024))) char ring[ST * T::kStage];
  const BwdSched& sc = p.sched[KV ? 1 : 0];
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // an XCD takes a contiguous run of (batch, head, tile)
  const int nblk = gridDim.x, bid = blockIdx.x;
  const int xcd = bid & 7, kx = bid >> 3, per = nblk >> 3, rem = nblk & 7;
  const int w = xcd < rem ? xcd * (per + 1) + kx : rem * (per + 1) + (xcd - rem) * per + kx;
  const int bh = w / sc.n_tiles, t = w % sc.n_tiles;
  const int b = bh / p.H, h = bh % p.H;
  int si = 0;
  while (si + 1 < sc.n_seg && sc.seg[si + 1].tile0 <= t) ++si;
  const BwdSeg seg = sc.seg[si];
  const int own0 = (t - seg.tile0) * T::kOwn + wave * 32 * NB;  // inside the segment

  const int64_t o_st = int64_t(p.H) * D;
  const int64_t q_base = int64_t(b) * p.n_rows * p.st + int64_t(h) * D;
  const int64_t o_base = int64_t(b) * p.n_rows * o_st + int64_t(h) * D;
  const int64_t s_base = int64_t(bh) * p.n_rows;
  const uint16_t* x1 = (KV ? p.k : p.q) + q_base;
  const uint16_t* x2 = KV ? p.v + q_base : p.d_o + o_base;
  const int64_t x2_st = KV ? p.st : o_st;
  const uint16_t* y1 = (KV ? p.q : p.k) + q_base;
  const uint16_t* y2 = KV ? p.d_o + o_base : p.v + q_base;
  const int64_t y1_st = p.st, y2_st = KV ? o_st : p.st;

  // own operands: row lane % 32, d = 16 c + 8 hh .. +7
  bf16x8 f1[NB][DC], f2[NB][DC];
  f32x16 cs[NB], cd[NB];  // dQ: -lse/scale and -D of the lane's query, the products' first addends
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
      const float l = in ? p.nlse[s_base + row] : 0.f, d = in ? p.ndelta[s_base + row] : 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) cs[nb][i] = l, cd[nb][i] = d;
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

  // streamed tiles
  int n_tiles = 0;
  for (int i = 0; i < seg.nr; ++i) n_tiles += (sc.range[seg.r0 + i].len + kTile - 1) / kTile;
  int ir = seg.r0, it = 0;  // next tile to load: range, tile in it
  const uint32_t lds0 = lds_u32(ring);
  const auto issue = [&](uint32_t stage) {
    const bool any = ir < seg.r0 + seg.nr;
    const BwdRange rg = sc.range[any ? ir : 0];
    const int64_t row = any ? rg.start + int64_t(it) * kTile : 0;
    const int valid = any ? min(kTile, rg.len - it * kTile) : 0;
    const __amdgpu_buffer_rsrc_t r1 = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(y1 + row * y1_st), (short)0, __builtin_bit_cast(int, uint32_t(valid) * uint32_t(y1_st * 2)), 0x00020000);
    const __amdgpu_buffer_rsrc_t r2 = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(y2 + row * y2_st), (short)0, __builtin_bit_cast(int, uint32_t(valid) * uint32_t(y2_st * 2)), 0x00020000);
    constexpr int CH = kT / 1024 / NW;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int pz = (i * NW + wave) * 64 + lane, rr = pz / GR, g = (pz % GR) ^ swz(rr, GR);
      dma16(lds0 + stage + (i * NW + wave) * 1024, uint32_t(rr) * uint32_t(y1_st * 2) + g * 16, r1);
      dma16(lds0 + stage + kT + (i * NW + wave) * 1024, uint32_t(rr) * uint32_t(y2_st * 2) + g * 16, r2);
    }
    if constexpr (KV) {
      const __amdgpu_buffer_rsrc_t rl = __builtin_amdgcn_make_buffer_rsrc(
          (void*)((wave & 1 ? p.ndelta : p.nlse) + s_base + row), (short)0, valid * 4, 0x00020000);
      dma4(lds0 + stage + 2 * kT + (wave & 1) * 256, lane * 4, rl);
    }
    if (any && ++it * kTile >= rg.len) ++ir, it = 0;
  };
  constexpr int kLoads = 2 * (kT / 1024 / NW) + (KV ? 1 : 0);
#pragma unroll
  for (int s = 0; s < ST - 1; ++s) issue(s * T::kStage);

  // fragment addresses
  const int li = lane & 15;
  const uint32_t fk = (lane & 31) * D * 2 + 16 * (swz(lane & 31, GR) ^ hh);
  const int gc = 2 * ((lane >> 4) & 1) + ((li & 3) >> 1);
  const int r0 = 4 * hh + (li >> 2), r1 = r0 + 8;
  const uint32_t v0 = r0 * D * 2 + 16 * (gc ^ swz(r0, GR)) + 8 * (li & 1);
  const uint32_t v1 = r1 * D * 2 + 16 * (gc ^ swz(r1, GR)) + 8 * (li & 1);

  int cr = seg.r0, ct = 0;
  uint32_t cur = 0, fill = (ST - 1) * T::kStage;
  for (int tile = 0; tile < n_tiles; ++tile) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 2) * kLoads) : "memory");
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    issue(fill);
    const int valid = min(kTile, sc.range[cr].len - ct * kTile);
    if (++ct * kTile >= sc.range[cr].len) ++cr, ct = 0;
    const char* st = ring + cur;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x16 s[NB], dp[NB];
      const char* a1 = st + j * 32 * D * 2;
      const char* a2 = a1 + kT;
      if constexpr (KV) {
        const char* sp = st + 2 * kT + j * 128 + hh * 16;
        f32x16 l, d;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(sp + g * 32);
          const f32x4 y = *reinterpret_cast<const f32x4*>(sp + 256 + g * 32);
#pragma unroll
          for (int e = 0; e < 4; ++e) l[4 * g + e] = x[e], d[4 * g + e] = y[e];
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb] = l, dp[nb] = d;
      } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb] = cs[nb], dp[nb] = cd[nb];
      }
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(a1 + (fk ^ uint32_t(32 * c)));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, f1[nb][c], s[nb], 0, 0, 0);
      }
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(a2 + (fk ^ uint32_t(32 * c)));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) dp[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, f2[nb][c], dp[nb], 0, 0, 0);
      }
      if (valid < 32 * (j + 1)) {
        const int lim = valid - 32 * j - 4 * hh;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (8 * (r >> 2) + (r & 3) >= lim) s[nb][r] = -INFINITY;
      }
      bf16x8 pf[NB][2], df[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(s[nb][r] * p.scale_log2);
          if constexpr (KV) pf[nb][r >> 3][r & 7] = (__bf16)e;
          df[nb][r >> 3][r & 7] = (__bf16)(e * dp[nb][r]);
        }
#pragma unroll
      for (int f = 0; f < 2 * DB; ++f) {
        const int ks = f / DB, d = f % DB;
        const auto tr = [&](const char* base) {
          const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base + ks * 16 * D * 2 + (v0 ^ uint32_t(64 * d))));
          const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base + ks * 16 * D * 2 + (v1 ^ uint32_t(64 * d))));
          return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        const bf16x8 a = tr(a1);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          acc1[nb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, df[nb][ks], acc1[nb][d], 0, 0, 0);
        if constexpr (KV) {
          const bf16x8 e = tr(a2);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            acc2[nb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(e, pf[nb][ks], acc2[nb][d], 0, 0, 0);
        }
      }
    }
    cur = cur + T::kStage == ST * T::kStage ? 0 : cur + T::kStage;
    fill = fill + T::kStage == ST * T::kStage ? 0 : fill + T::kStage;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the work-group

  const auto store = [&](uint16_t* out, const f32x16& acc, int nb, int d, float f) {
    const int r = own0 + nb * 32 + (lane & 31);
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
      if (r < seg.len)
        *reinterpret_cast<bf16x8*>(out + (int64_t(b) * p.n_rows + seg.row0 + r) * p.g_st + int64_t(h) * D + d * 32 +
                                   16 * i + 8 * hh) = o;
    }
  };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      store(KV ? p.dk : p.dq, acc1[nb][d], nb, d, p.scale);
      if constexpr (KV) store(p.dv, acc2[nb][d], nb, d, 1.f);
    }
}

// -lse / scale and -D of every row; rows that read nothing get -inf and 0.
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

#ifndef BWD_NB
#define BWD_NB 1
#endif
template <int D>
void launch(const BwdParams& p, hipStream_t s) {
  const int64_t rows = int64_t(p.B) * p.n_rows * p.H;
  hipLaunchKernelGGL(attn_bwd_rows_kernel<D>, dim3((rows * (D / 8) + 255) / 256), dim3(256), 0, s, p);
  const int64_t bh = int64_t(p.B) * p.H;
  constexpr int NB = BWD_NB, NW = kBwdOwn / 32 / NB, ST = 3;
  hipLaunchKernelGGL((attn_bwd_kernel<D, true, NB, NW, ST>), dim3(bh * p.sched[1].n_tiles), dim3(64 * NW), 0, s, p);
  hipLaunchKernelGGL((attn_bwd_kernel<D, false, NB, NW, ST>), dim3(bh * p.sched[0].n_tiles), dim3(64 * NW), 0, s, p);
}

}  // namespace

int launch_attention_bwd(const BwdParams& p, int D, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64) launch<64>(p, s);
  else launch<128>(p, s);
  return int(hipGetLastError());
}

}  // namespace rc
