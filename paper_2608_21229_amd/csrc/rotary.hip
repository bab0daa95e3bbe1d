// Queries and keys: RMS norm of each head row (optional), then a rotation of
// its channel pairs by the token's position on several axes.
//   z = w x r, r = rsqrt(mean x^2 + eps);  (a, b) -> (a cos t - b sin t, a sin t + b cos t),
//   t = position[axis of the pair] * frequency of the pair
// Backward: u is the gradient turned back; with a norm, xh = x r:
//   dx = r (u w - xh mean(u w xh)),  dw = sum over all rows of u xh
//
// The norm's sums and the rotation are fp32 (angles reduced in 64 bits); each
// output is rounded once.
//
// HBM-bound: every row is read and written once: 4608 tokens of 24 heads, D = 128,
// with the norm 20 us (113 MB, partly from cache; 24 with six sets of rows in turn); 2 x
// 7801 tokens of 12 heads backward 71 us (288 MB, 4.1 TB/s) and 5 us for dw.  A head row is D / 8 lanes of 16
// bytes, so a wave holds 512 / D head rows; it takes a token's rows of one
// tensor after another, kAhead loads in flight, with the token's sines and
// cosines (and the norm's weights) in registers.  out[e] = r (x[e] A[e] + x'[e] B[e])
// with x' the partner channel: of the lane itself, or of the lane that holds the
// other half.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_lanes.h"
#include "rc_layer.h"

namespace rc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kAhead = 4;  // row groups loaded together

__device__ __forceinline__ u32x4 load16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }
// Past the caches go the stores of rotary_kernel (the forward, and the gradient without
// a norm) and the loads of the gradient with a norm (new rows each call: a step's
// rotation 23.1 -> 20.3 us, the video's gradient 81.9 -> 73.9; the other loads and
// stores gained nothing or lost).  Between the calls that write and read the rows it makes
// no difference: projection, rotation and attention of a step 574 us with and 573
// without, attention gradient, rotation gradient and projection of 8768 tokens of 20 heads
// 2020 and 2016, without a norm 1984 and 1983.  A gradient called again on rows that the
// last-level cache would have kept loses: 4608 tokens of 24 heads 36 -> 41.
__device__ __forceinline__ u32x4 load16_once(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}
template <bool ONCE>
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (__bf16)v[e];
  if constexpr (ONCE) __builtin_nontemporal_store(o, reinterpret_cast<bf16x8*>(p));
  else *reinterpret_cast<bf16x8*>(p) = o;
}
__device__ __forceinline__ void unpack(u32x4 raw, float (&v)[8]) {
  const bf16x8 b = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = float(b[e]);
}

// Which lane holds the partner channels, in bytes of a lane index (halves).
template <int D>
__device__ __forceinline__ int partner(const RotaryParams& p, int lane, int g) {
  const int hg = p.half / 8;
  return 4 * (lane + (g < hg ? hg : g < 2 * hg ? -hg : 0));
}
// Whether the pair of a granule's channel e turns (with halves a granule turns
// as a whole).  The channels past the rotated width stay what they are, whatever
// else the row holds: a partner of zero, A = 1 and B = -0 for them.
template <bool HALVES>
__device__ __forceinline__ bool turns(const RotaryParams& p, int g, int e) {
  return g * 8 + (HALVES ? 0 : e & ~1) < p.width;
}
template <bool HALVES>
__device__ __forceinline__ void partners(const RotaryParams& p, u32x4 raw, const float (&v)[8], int g, int from,
                                         float (&o)[8]) {
  if constexpr (HALVES) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = __builtin_amdgcn_ds_bpermute(from, int(raw[i]));
      if (!turns<HALVES>(p, g, 0)) r[i] = 0;
    }
    unpack(r, o);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = turns<HALVES>(p, g, e) ? v[e ^ 1] : 0.f;
  }
}

// A = cos, B = -sin or sin of the lane's channels.  A turn is the position times
// the frequency in 64 bits (far positions lose their fraction in 32), reduced
// to half a revolution either way; v_sin and v_cos take revolutions.
template <bool HALVES>
__device__ __forceinline__ void angles(const RotaryParams& p, int64_t tok, int g, float (&A)[8], float (&B)[8]) {
  const int64_t b = tok / p.N, n = tok - b * p.N;
  const char* pos = static_cast<const char*>(p.pos) + 4 * (b * p.pos_sb + n * p.axes);
  constexpr int NP = HALVES ? 8 : 4;
  float c[NP], s[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int ch = g * 8 + i;
    const int pair = HALVES ? (ch < p.half ? ch : ch < 2 * p.half ? ch - p.half : 63) : g * 4 + i;
    const double f = HALVES && ch >= 2 * p.half ? 0.0 : p.turns[pair];
    const char* at = pos + 4 * p.axis[pair];
    double t = p.pos_float ? double(*reinterpret_cast<const float*>(at)) : double(*reinterpret_cast<const int32_t*>(at));
    t *= f;
    t -= rint(t);
    c[i] = __builtin_amdgcn_cosf(float(t));
    s[i] = __builtin_amdgcn_sinf(float(t)) * p.sign;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    A[e] = c[HALVES ? e : e / 2];
    B[e] = HALVES ? (g * 8 < p.half ? -s[HALVES ? e : 0] : s[HALVES ? e : 0]) : e & 1 ? s[e / 2] : -s[e / 2];
    if (!turns<HALVES>(p, g, e)) A[e] = 1.f, B[e] = -0.f;
  }
}

// Weight of each channel into A, of its partner into B.
template <bool HALVES>
__device__ __forceinline__ void weigh(const RotaryParams& p, const uint16_t* w, int g, int from, float (&A)[8],
                                      float (&B)[8]) {
  const u32x4 raw = load16(w + g * 8);
  float v[8], o[8];
  unpack(raw, v);
  partners<HALVES>(p, raw, v, g, from, o);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    A[e] *= v[e];
    B[e] *= o[e];
  }
}

template <int D, bool HALVES>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
  constexpr int L = D / 8, RW = 64 / L;  // lanes per head row, head rows per wave
  const int lane = threadIdx.x & 63, g = lane % L, sub = lane / L;
  const int per = (p.H + RW - 1) / RW, both = p.x[0] && p.x[1] ? 2 * per : per;  // row groups of a tensor, of a token
  const uint32_t splits = (both + p.groups - 1) / p.groups;
  const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tok = unit / splits;
  if (tok >= p.N * p.B) return;
  const int end = min(both, int(unit % splits + 1) * p.groups);
  const int from = HALVES ? partner<D>(p, lane, g) : 0;
  float A[8], B[8], cA[8], cB[8];
  int have = -1;
  for (int i0 = int(unit % splits) * p.groups; i0 < end;) {
    const int k = !p.x[0] || i0 >= per ? 1 : 0;  // queries, then keys
    const uint16_t* x = (k ? p.x[1] : p.x[0]) + tok * p.x_st + g * 8;
    uint16_t* y = (k ? p.y[1] : p.y[0]) + tok * p.y_st + g * 8;
    const uint16_t* w = k ? p.w[1] : p.w[0];
    const int first = k && p.x[0] ? i0 - per : i0;
    const int stop = min(first + end - i0, per);
    for (int j0 = first; j0 < stop; j0 += kAhead) {
      u32x4 raw[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int h = min((j0 + j) * RW + sub, p.H - 1);
        if (j0 + j < stop) raw[j] = load16(x + int64_t(h) * D);
      }
      if (have < 0) angles<HALVES>(p, tok, g, A, B);
      if (have != k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) cA[e] = A[e], cB[e] = B[e];
        if (w) weigh<HALVES>(p, w, g, from, cA, cB);
        have = k;
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (j0 + j >= stop) continue;
        float v[8], o[8], r = 1.f;
        unpack(raw[j], v);
        partners<HALVES>(p, raw[j], v, g, from, o);
        if (w) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += v[e] * v[e];
          r = rsqrtf(group_sum<L>(ss) * (1.f / D) + p.eps);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = r * (v[e] * cA[e] + o[e] * cB[e]);
        const int h = (j0 + j) * RW + sub;
        if (h < p.H) store8<true>(y + int64_t(h) * D, v);
      }
    }
    i0 += stop - first;
  }
}

// Backward with a norm: a work-group takes a contiguous run of tokens, its
// waves every fourth of them, and leaves its sums of dw.  Three work-groups per CU
// (their registers' limit): 4608 x 24 and 15602 x 12 head rows take 41.4 and 61.5 us with
// 768, 51.9 and 79.4 with 256, 55.2 and 72.7 with 1024, whose last 256 run alone.
template <int D, bool HALVES>
__global__ __launch_bounds__(256, 3) void rotary_norm_backward_kernel(const RotaryParams p) {
  constexpr int L = D / 8, RW = 64 / L;
  __shared__ float sums[4][2][D];
  const int lane = threadIdx.x & 63, g = lane % L, sub = lane / L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t toks = p.N * p.B;
  const int64_t t0 = toks * blockIdx.x / p.blocks, t1 = toks * (blockIdx.x + 1) / p.blocks;
  const int per = (p.H + RW - 1) / RW;
  const int from = HALVES ? partner<D>(p, lane, g) : 0;
  float dw[2][8];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[k][e] = 0.f;
  for (int64_t tok = t0 + wave; tok < t1; tok += 4) {
    float A[8], B[8];
    bool have = false;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!p.x[k]) continue;
      const uint16_t* w = p.w[k];
      const uint16_t* gr = p.x[k] + tok * p.x_st + g * 8;
      const uint16_t* xr = w ? p.n[k] + tok * p.n_st + g * 8 : gr;
      uint16_t* y = p.y[k] + tok * p.y_st + g * 8;
      for (int j0 = 0; j0 < per; j0 += kAhead) {
        u32x4 rg[kAhead], rx[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (j0 + j >= per) continue;
          const int64_t at = int64_t(min((j0 + j) * RW + sub, p.H - 1)) * D;
          rg[j] = load16_once(gr + at);
          if (w) rx[j] = load16_once(xr + at);
        }
        if (!have) angles<HALVES>(p, tok, g, A, B);
        have = true;
        float wv[8];
        if (w) unpack(load16(w + g * 8), wv);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (j0 + j >= per) continue;
          const int h = (j0 + j) * RW + sub;
          float u[8], o[8];
          unpack(rg[j], u);
          partners<HALVES>(p, rg[j], u, g, from, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = u[e] * A[e] + o[e] * B[e];
          if (w) {
            float x[8], ss = 0.f, dot = 0.f;
            unpack(rx[j], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              u[e] = o[e] * wv[e];
              ss += x[e] * x[e];
              dot += u[e] * x[e];
            }
            const float r = rsqrtf(group_sum<L>(ss) * (1.f / D) + p.eps);
            const float m = group_sum<L>(dot) * (1.f / D) * r * r;
            if (h < p.H) {  // the lanes past the last head hold its row once more
#pragma unroll
              for (int e = 0; e < 8; ++e) dw[k][e] += o[e] * (x[e] * r);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = r * (u[e] - x[e] * m);
          }
          if (h < p.H) store8<false>(y + int64_t(h) * D, o);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = dw[k][e];
#pragma unroll
      for (int m = L; m < 64; m <<= 1) x += __shfl_xor(x, m);
      if (sub == 0) sums[wave][k][g * 8 + e] = x;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += 256) {
    const int k = i / D, c = i % D;
    p.partial[int64_t(blockIdx.x) * 2 * D + i] = (sums[0][k][c] + sums[1][k][c]) + (sums[2][k][c] + sums[3][k][c]);
  }
}

// dw from the work-groups' sums: 16 columns per work-group, 64 threads each,
// eight loads in flight; every column's sum keeps one order.
template <int D>
__global__ __launch_bounds__(1024) void rotary_dw_kernel(const RotaryParams p) {
  __shared__ float part[64][17];
  const int c = threadIdx.x & 15, s = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float x = 0.f;
  for (int i = s; i < p.blocks; i += 64 * 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = i + 64 * j;
      v[j] = at < p.blocks ? p.partial[int64_t(at) * 2 * D + col] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x += v[j];
  }
  part[s][c] = x;
  __syncthreads();
  if (s >= 4) return;  // one wave: four threads per column
  x = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) x += part[s * 16 + i][c];
  x += __shfl_xor(x, 16);
  x += __shfl_xor(x, 32);
  float* dw = p.dw[col / D];
  if (dw && s == 0) dw[col % D] = x;
}

template <int D>
void launch(const RotaryParams& p, hipStream_t s) {
  constexpr int RW = 512 / D;
  const int per = (p.H + RW - 1) / RW, both = p.x[0] && p.x[1] ? 2 * per : per;
  const int splits = (both + p.groups - 1) / p.groups;
  const dim3 grid((p.N * p.B * splits + 3) / 4);
  if (p.half > 0) hipLaunchKernelGGL((rotary_kernel<D, true>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((rotary_kernel<D, false>), grid, dim3(256), 0, s, p);
}

template <int D>
void launch_norm_bwd(const RotaryParams& p, hipStream_t s) {
  if (p.half > 0) hipLaunchKernelGGL((rotary_norm_backward_kernel<D, true>), dim3(p.blocks), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((rotary_norm_backward_kernel<D, false>), dim3(p.blocks), dim3(256), 0, s, p);
  hipLaunchKernelGGL(rotary_dw_kernel<D>, dim3(2 * D / 16), dim3(1024), 0, s, p);
}

}  // namespace

int launch_rotary(const RotaryParams& p, int D, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64) launch<64>(p, s);
  else launch<128>(p, s);
  return int(hipGetLastError());
}

int launch_rotary_norm_backward(const RotaryParams& p, int D, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64) launch_norm_bwd<64>(p, s);
  else launch_norm_bwd<128>(p, s);
  return int(hipGetLastError());
}

}  // namespace rc
