// Queries and keys: RMS norm of each head row (optional), then a rotation of
// its channel pairs by the token's position on several axes.
//   z = w x rsqrt(mean x^2 + eps);  (a, b) -> (a cos t - b sin t, a sin t + b cos t),
//   t = position[axis of the pair] * frequency of the pair
// Backward: u is the gradient turned back; with a norm, xh = x r:
//   dx = r (u w - xh mean(u w xh)),  dw = sum over all rows of u xh
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_layer.h"

namespace rc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Angles {
  float c[8], s[8];  // of the lane's 8 channels (halves), or of its 4 pairs
};

// The turn of a pair in 64 bits (far positions lose their fraction in 32),
// reduced to half a revolution either way; v_sin and v_cos take revolutions.
template <int D, bool HALVES>
__device__ __forceinline__ Angles angles(const RotaryParams& p, int64_t b, int64_t n, int g) {
  Angles a;
  const char* pos = static_cast<const char*>(p.pos) + 4 * (b * p.pos_sb + n * p.axes);
  constexpr int NP = HALVES ? 8 : 4;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    int pair = g * NP + i;
    if (HALVES) pair = pair < p.half ? pair : pair < 2 * p.half ? pair - p.half : 63;
    const double turn = HALVES && g * 8 + i >= 2 * p.half ? 0.0 : p.turns[pair];
    const char* at = pos + 4 * p.axis[pair];
    const double x = p.pos_float ? double(*reinterpret_cast<const float*>(at)) : double(*reinterpret_cast<const int32_t*>(at));
    double t = x * turn;
    t -= rint(t);
    a.c[i] = __builtin_amdgcn_cosf(float(t));
    a.s[i] = __builtin_amdgcn_sinf(float(t)) * p.sign;
  }
  return a;
}

// Sum over the lanes of a head row.
template <int L>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int m = L / 2; m > 0; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

template <int D, bool HALVES>
__device__ __forceinline__ void turn(const RotaryParams& p, const Angles& a, int g, float (&v)[8]) {
  if (HALVES) {
    const int hg = p.half / 8;
    const int other = g < hg ? g + hg : g < 2 * hg ? g - hg : g;
    const float sg = g < hg ? -1.f : 1.f;
    const int lane = threadIdx.x & 63, src = lane - g + other;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __shfl(v[i], src);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] * a.c[i] + sg * w[i] * a.s[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = v[2 * i], y = v[2 * i + 1];
      v[2 * i] = x * a.c[i] - y * a.s[i];
      v[2 * i + 1] = x * a.s[i] + y * a.c[i];
    }
  }
}

template <int D, bool HALVES, bool NORM>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
  constexpr int L = D / 8, RW = 64 / L;  // lanes per head row, head rows per wave
  const int lane = threadIdx.x & 63, g = lane % L, sub = lane / L;
  const int rows = (p.x[0] ? p.H : 0) + (p.x[1] ? p.H : 0);  // head rows of a token
  const int per_tok = ((rows + RW - 1) / RW + p.groups - 1) / p.groups;
  const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t tok = unit / per_tok;
  if (tok >= p.N * p.B) return;
  const int first = int(unit % per_tok) * p.groups;
  const int64_t b = tok / p.N, n = tok % p.N;
  const Angles a = angles<D, HALVES>(p, b, n, g);
  for (int i = 0; i < p.groups; ++i) {
    const int r = (first + i) * RW + sub;
    const bool in = r < rows;
    const bool which = in ? !p.x[0] || r >= p.H : !p.x[0];  // keys
    const int h = in ? (p.x[0] && which ? r - p.H : r) : 0;
    const uint16_t* x = (which ? p.x[1] : p.x[0]) + tok * p.x_st + int64_t(h) * D + g * 8;
    const bf16x8 raw = *reinterpret_cast<const bf16x8*>(x);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(raw[e]);
    if (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += v[e] * v[e];
      const float rr = rsqrtf(row_sum<L>(ss) * (1.f / D) + p.eps);
      const uint16_t* wp = which ? p.w[1] : p.w[0];
      if (wp) {
        const bf16x8 w = *reinterpret_cast<const bf16x8*>(wp + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * rr * float(w[e]);
      }
    }
    turn<D, HALVES>(p, a, g, v);
    if (in) {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (__bf16)v[e];
      *reinterpret_cast<bf16x8*>((which ? p.y[1] : p.y[0]) + tok * p.y_st + int64_t(h) * D + g * 8) = o;
    }
  }
}

// Backward with a norm: a work-group takes a contiguous run of tokens, its
// waves every fourth of them, and leaves its sums of dw.
template <int D, bool HALVES>
__global__ __launch_bounds__(256) void rotary_norm_backward_kernel(const RotaryParams p) {
  constexpr int L = D / 8, RW = 64 / L;
  __shared__ float sums[4][2][D];
  const int lane = threadIdx.x & 63, g = lane % L, sub = lane / L, wave = threadIdx.x >> 6;
  const int64_t toks = p.N * p.B;
  const int64_t t0 = toks * blockIdx.x / p.blocks, t1 = toks * (blockIdx.x + 1) / p.blocks;
  float dw[2][8];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[k][e] = 0.f;
  for (int64_t tok = t0 + wave; tok < t1; tok += 4) {
    const Angles a = angles<D, HALVES>(p, tok / p.N, tok % p.N, g);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!p.x[k]) continue;
      float w[8];
      if (p.w[k]) {
        const bf16x8 raw = *reinterpret_cast<const bf16x8*>(p.w[k] + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = float(raw[e]);
      }
      for (int h0 = 0; h0 < p.H; h0 += RW) {
        const bool in = h0 + sub < p.H;
        const int64_t at = int64_t(in ? h0 + sub : 0) * D + g * 8;
        const bf16x8 rg = *reinterpret_cast<const bf16x8*>(p.x[k] + tok * p.x_st + at);
        float u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = float(rg[e]);
        turn<D, HALVES>(p, a, g, u);
        if (p.w[k]) {
          const bf16x8 rx = *reinterpret_cast<const bf16x8*>(p.n[k] + tok * p.n_st + at);
          float x[8], ss = 0.f, dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = float(rx[e]);
            ss += x[e] * x[e];
            dot += u[e] * w[e] * x[e];
          }
          const float rr = rsqrtf(row_sum<L>(ss) * (1.f / D) + p.eps);
          const float m = row_sum<L>(dot) * (1.f / D) * rr * rr;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (in) dw[k][e] += u[e] * x[e] * rr;
            u[e] = rr * (u[e] * w[e] - x[e] * m);
          }
        }
        if (in) {
          bf16x8 o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (__bf16)u[e];
          *reinterpret_cast<bf16x8*>(p.y[k] + tok * p.y_st + at) = o;
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

// dw from the work-groups' sums: 32 columns per work-group, 32 threads each.
template <int D>
__global__ __launch_bounds__(1024) void rotary_dw_kernel(const RotaryParams p) {
  __shared__ float part[32][33];
  const int c = threadIdx.x & 31, s = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  float x = 0.f;
  for (int i = s; i < p.blocks; i += 32) x += p.partial[int64_t(i) * 2 * D + col];
  part[s][c] = x;
  __syncthreads();
  if (s != 0) return;
  x = 0.f;
  for (int i = 0; i < 32; ++i) x += part[i][c];
  float* dw = p.dw[col / D];
  if (dw) dw[col % D] = x;
}

template <int D>
void launch(const RotaryParams& p, hipStream_t s) {
  constexpr int RW = 512 / D;
  const int rows = (p.x[0] ? p.H : 0) + (p.x[1] ? p.H : 0);
  const int per_tok = ((rows + RW - 1) / RW + p.groups - 1) / p.groups;
  const dim3 grid((p.N * p.B * per_tok + 3) / 4);
  const bool norm = p.w[0] || p.w[1];
  if (p.half > 0) {
    if (norm) hipLaunchKernelGGL((rotary_kernel<D, true, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((rotary_kernel<D, true, false>), grid, dim3(256), 0, s, p);
  } else {
    if (norm) hipLaunchKernelGGL((rotary_kernel<D, false, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((rotary_kernel<D, false, false>), grid, dim3(256), 0, s, p);
  }
}

template <int D>
void launch_norm_bwd(const RotaryParams& p, hipStream_t s) {
  if (p.half > 0) hipLaunchKernelGGL((rotary_norm_backward_kernel<D, true>), dim3(p.blocks), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((rotary_norm_backward_kernel<D, false>), dim3(p.blocks), dim3(256), 0, s, p);
  hipLaunchKernelGGL(rotary_dw_kernel<D>, dim3(2 * D / 32), dim3(1024), 0, s, p);
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
