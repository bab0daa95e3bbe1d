// Gated norm between two blocks of a layer: the residual with the block's
// gated output, then the norm and modulation that the next block reads.
//   u  = x, or w_p x rsqrt(mean x^2 + eps)
//   h' = h + a gate u
//   y  = n(h') w (1 + scale) + shift,  n the layer norm without affine, or the RMS norm
// gate, scale and shift belong to a row's group (one vector per batch entry and
// group).  Backward, with x^ = n(h') before w and r its reciprocal deviation:
//   dn = dy w (1 + scale);  dh = dh' + r (dn - mean(dn) - x^ mean(dn x^))   (RMS: without mean(dn))
//   dx = a gate w_p dh, through the norm of x the same way
//   dshift = sum dy, dscale = w sum dy x^, dgate = a sum dh u over a group's rows
// Rows are bf16 and everything computed from them fp32, the means in a second
// pass over the registers (the row is in them); each output is rounded once.
//
// HBM-bound: every row is read once and written once.  4608 rows of 2560 channels
// forward 17 us (94 MB, partly from cache; 20 with six sets of rows in turn); 8768 rows
// backward 61 us (269 MB, 4.4 TB/s) and 6.5 us for the gradients shared by the rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_lanes.h"
#include "rc_layer.h"

namespace rc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bf16x8 load8(const uint16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
// What is not read again soon does not stay in the caches: the forward's h', which the
// next residual reads, and the gradient's loads, also behind the projection that wrote dy
// and before the one that reads dx (8768 rows of 2560: 494 -> 487 us for the three; new
// rows each call, alone: 73.6 -> 68.3).  y stays, since a projection reads it next: norm
// and projection of 4608 rows of 2560 take 173 us, 186 with y past the caches, two layers'
// recompute of 8768 rows 2139 and 2168, though the norm alone then takes 20.4, not 19.5.
// The forward's loads and the gradient's stores gained nothing or lost.  A gradient
// called again on rows that the last-level cache would have kept loses: 10877 rows of
// 1928 57 -> 65.
__device__ __forceinline__ bf16x8 load8_once(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(p));
}
template <bool ONCE>
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (__bf16)v[e];
  if constexpr (ONCE) __builtin_nontemporal_store(o, reinterpret_cast<bf16x8*>(p));
  else *reinterpret_cast<bf16x8*>(p) = o;
}

// Sums over the T threads of a row.  Each array has two halves that take turns,
// so that one barrier per sum is enough: a half is written again only after
// the next sum's barrier, which every reader of it has reached.
template <int K>
struct RowSums {
  float at[2][16][K];
};
template <int T, int K>
__device__ __forceinline__ void row_sums(float (&x)[K], RowSums<K>& lds, int row, int& half) {
#pragma unroll
  for (int k = 0; k < K; ++k) x[k] = wave_sum(x[k]);
  if constexpr (T > 64) {
    constexpr int W = T / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) lds.at[half][wave][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += lds.at[half][row * W + w][k];
      x[k] = s;
    }
    half ^= 1;
  }
}

__device__ __forceinline__ int group_of(const NormParams& p, int n) {
  int s = 0;
  while (s + 1 < p.n_spans && p.span_row0[s + 1] <= n) ++s;
  return p.span_group[s];
}

// T threads per row, GP granules of 8 channels per thread.
template <int T, int GP>
__global__ __launch_bounds__(256) void norm_kernel(const NormParams p) {
  __shared__ RowSums<1> lds;
  constexpr int RB = 256 / T;
  const int t = threadIdx.x % T, rb = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
  const uint32_t N = uint32_t(p.N), r_ = blockIdx.x * RB + rb;
  const bool in = r_ < N * p.B;
  const uint32_t r32 = in ? r_ : 0, b = r32 / N;
  const int64_t r = r32;
  const int64_t mod = b * p.mod_sb + int64_t(group_of(p, int(r32 - b * N))) * p.mod_sg;
  const int ng = p.C / 8;
  int half = 0;
  float h[GP][8];
#pragma unroll
  for (int i = 0; i < GP; ++i) {
    const int g = t + i * T;
    const bool has = g < ng;
    const bf16x8 a = has ? load8(p.h.p + r * p.h.ld + g * 8) : bf16x8{};
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = float(a[e]);
  }
  if (p.x.p) {
    float x[GP][8], k[1] = {1.f};
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const int g = t + i * T;
      const bf16x8 a = g < ng ? load8(p.x.p + r * p.x.ld + g * 8) : bf16x8{};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = float(a[e]);
    }
    if (p.post) {
      k[0] = 0.f;
#pragma unroll
      for (int i = 0; i < GP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) k[0] += x[i][e] * x[i][e];
      row_sums<T, 1>(k, lds, rb, half);
      k[0] = rsqrtf(k[0] * p.inv_c + p.eps);
    }
    const float f = k[0] * p.rscale;
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const int g = t + i * T;
      if (g >= ng) continue;
      if (p.post_weight) {
        const bf16x8 w = load8(p.post_weight + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] *= float(w[e]);
      }
      if (p.gate) {
        const bf16x8 w = load8(p.gate + mod + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] *= float(w[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += f * x[i][e];
      if (in) store8<true>(p.h_out.p + r * p.h_out.ld + g * 8, h[i]);
    }
  }
  if (!p.y.p) return;
  if (!p.rms) {
    float m[1] = {0.f};
#pragma unroll
    for (int i = 0; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m[0] += h[i][e];
    row_sums<T, 1>(m, lds, rb, half);
    const float mean = m[0] * p.inv_c;
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      if (t + i * T >= ng) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] -= mean;
    }
  }
  float v[1] = {0.f};
#pragma unroll
  for (int i = 0; i < GP; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[0] += h[i][e] * h[i][e];
  row_sums<T, 1>(v, lds, rb, half);
  const float rs = rsqrtf(v[0] * p.inv_c + p.eps);
#pragma unroll
  for (int i = 0; i < GP; ++i) {
    const int g = t + i * T;
    if (g >= ng) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] *= rs;
    if (p.weight) {
      const bf16x8 w = load8(p.weight + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] *= float(w[e]);
    }
    if (p.scale) {
      const bf16x8 w = load8(p.scale + mod + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += h[i][e] * float(w[e]);
    }
    if (p.shift) {
      const bf16x8 w = load8(p.shift + mod + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += float(w[e]);
    }
    if (in) store8<false>(p.y.p + r * p.y.ld + g * 8, h[i]);
  }
}

// Backward: a work-group of 512 threads takes one chunk of rows of one batch
// entry and span, NT / T rows at a time, and leaves the chunk's sums over its
// rows of dy, dy n and dh' x^ (the gradients of shift, scale and gate up to
// factors of the column).  The chunk's vectors (1 + scale) w and a gate w_p lie in
// LDS; the next rows are loaded before the present ones are computed, except
// with 4 granules a thread, whose registers that would overflow (1280 rows of 16384
// channels: 144 us, 90 without; with the present loads 84).  The vectors' planes, and
// zeros of their own for lanes past a row's end, leave few LDS bank conflicts (two samples'
// 3936 rows of 1928 channels: 7.7 M -> 0.9 M -> 0.05 M cycles; 59.6 -> 52.9 us with the
// sums, then 57.7 -> 56.7 with new rows each call).
template <int T, int GP>
__global__ __launch_bounds__(512) void norm_backward_kernel(const NormParams p) {
  constexpr int NT = 512;
  constexpr bool kAhead = GP < 4;
  __shared__ RowSums<1> lds1;
  __shared__ RowSums<3> lds3;
  // two vectors (at the end the row groups' sums): the first four channels of all
  // granules, then the others, so that lanes next to each other read 16 bytes next to each other
  constexpr int kPlane = T * GP * 4;
  __shared__ __attribute__((aligned(16))) float vec[4 * kPlane];
  const auto at_vec = [](int g, int e) { return (e >> 2) * kPlane + g * 4 + (e & 3); };
  constexpr int RB = NT / T;
  const int t = threadIdx.x % T, rb = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
  const int64_t b = blockIdx.x / p.chunks;
  const int chunk = blockIdx.x % p.chunks;
  int sp = 0;
  while (sp + 1 < p.n_spans && p.span_chunk0[sp + 1] <= chunk) ++sp;
  const int first = (chunk - p.span_chunk0[sp]) * p.chunk_rows;
  const int count = min(p.chunk_rows, p.span_rows[sp] - first);
  const int64_t row0 = b * p.N + p.span_row0[sp] + first;
  const int64_t mod = b * p.mod_sb + int64_t(p.span_group[sp]) * p.mod_sg;
  const int ng = p.C / 8;
  bool has[GP];
#pragma unroll
  for (int i = 0; i < GP; ++i) has[i] = t + i * T < ng;

  const bool dy_ = p.dy.p != nullptr, dh_ = p.dh.p != nullptr, x_ = p.x.p != nullptr;
  bf16x8 ry[GP], rn[GP], rh[GP], rx[GP];  // the rows of the next step
  const auto load_rows = [&](int i0) {
    const int64_t r = row0 + i0 + rb;
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const int c = (t + i * T) * 8;
      ry[i] = rn[i] = rh[i] = rx[i] = bf16x8{};
      if (!has[i] || i0 + rb >= count) continue;  // zeros past the row's end and the chunk's
      if (dy_) {
        rn[i] = load8_once(p.h.p + r * p.h.ld + c);
        ry[i] = load8_once(p.dy.p + r * p.dy.ld + c);
      }
      if (dh_) rh[i] = load8_once(p.dh.p + r * p.dh.ld + c);
      if (x_) rx[i] = load8_once(p.x.p + r * p.x.ld + c);
    }
  };
  if constexpr (kAhead) load_rows(0);
  for (int g = threadIdx.x; g < T * GP; g += NT) {  // zeros past the row's end, where its values are zeros, too
    float s[8] = {}, a[8] = {};
    if (g < ng) {
      const bf16x8 vs = p.scale ? load8(p.scale + mod + g * 8) : bf16x8{};
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 1.f + float(vs[e]), a[e] = p.rscale;
      const auto times = [&](float (&v)[8], const uint16_t* w) {
        if (!w) return;
        const bf16x8 x = load8(w + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= float(x[e]);
      };
      times(s, p.weight);
      times(a, p.gate ? p.gate + mod : nullptr);
      times(a, p.post_weight);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) vec[at_vec(g, e)] = s[e], vec[2 * kPlane + at_vec(g, e)] = a[e];
  }
  __syncthreads();

  int half1 = 0, half3 = 0;
  float a_shift[GP][8], a_scale[GP][8], a_gate[GP][8];
#pragma unroll
  for (int i = 0; i < GP; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) a_shift[i][e] = a_scale[i][e] = a_gate[i][e] = 0.f;
  for (int i0 = 0; i0 < count; i0 += RB) {
    const bool in = i0 + rb < count;
    const int64_t r = row0 + i0 + rb;
    if constexpr (!kAhead) load_rows(i0);
    float n[GP][8], d[GP][8], dh[GP][8];
    bf16x8 cx[GP];
    float m[1] = {0.f};
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      cx[i] = rx[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[i][e] = float(rn[i][e]);
        d[i][e] = float(ry[i][e]);
        dh[i][e] = float(rh[i][e]);
        m[0] += n[i][e];
      }
    }
    if (kAhead && i0 + RB < count) load_rows(i0 + RB);
    if (dy_) {
      if (!p.rms) {
        row_sums<T, 1>(m, lds1, rb, half1);
        const float mean = m[0] * p.inv_c;
#pragma unroll
        for (int i = 0; i < GP; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) n[i][e] = has[i] ? n[i][e] - mean : 0.f;
      }
      // over the row: n^2, dn, dn n (dn = dy (1 + scale) w)
      float k[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < GP; ++i) {
        const float* w = vec + (t + i * T) * 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float dn = d[i][e] * w[at_vec(0, e)];
          k[0] += n[i][e] * n[i][e];
          k[1] += dn;
          k[2] += dn * n[i][e];
        }
      }
      row_sums<T, 3>(k, lds3, rb, half3);
      const float rs = rsqrtf(k[0] * p.inv_c + p.eps);
      const float mean = p.rms ? 0.f : k[1] * p.inv_c, dot = k[2] * p.inv_c * rs * rs;
      if (in) {  // a whole wave; rows past the chunk add nothing, whatever the vectors hold
#pragma unroll
        for (int i = 0; i < GP; ++i) {
          const float* w = vec + (t + i * T) * 4;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            a_shift[i][e] += d[i][e];
            a_scale[i][e] += d[i][e] * (n[i][e] * rs);
            dh[i][e] += rs * (d[i][e] * w[at_vec(0, e)] - mean - n[i][e] * dot);
          }
        }
      }
    }
    if (in) {
#pragma unroll
      for (int i = 0; i < GP; ++i)
        if (has[i]) store8<false>(p.dh_in.p + r * p.dh_in.ld + (t + i * T) * 8, dh[i]);
    }
    if (!x_) continue;
    float k[3] = {0.f, 0.f, 0.f}, rq = 1.f, dot = 0.f;
    if (p.post) {
#pragma unroll
      for (int i = 0; i < GP; ++i) {
        const float* w = vec + 2 * kPlane + (t + i * T) * 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = float(cx[i][e]);
          k[0] += x * x;
          k[1] += dh[i][e] * w[at_vec(0, e)] * x;
        }
      }
      row_sums<T, 3>(k, lds3, rb, half3);
      rq = rsqrtf(k[0] * p.inv_c + p.eps);
      dot = k[1] * p.inv_c * rq * rq;
    }
    if (!in) continue;
    const float gq = rq * p.rscale;
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const float* w = vec + 2 * kPlane + (t + i * T) * 4;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = float(cx[i][e]);
        a_gate[i][e] += dh[i][e] * (x * gq);
        o[e] = rq * (dh[i][e] * w[at_vec(0, e)] - x * dot);
      }
      if (has[i]) store8<false>(p.dx.p + r * p.dx.ld + (t + i * T) * 8, o);
    }
  }
  // the row groups' sums, in order, through LDS
  float* out = p.partial + int64_t(blockIdx.x) * 3 * p.C;
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    auto& a = q == 0 ? a_shift : q == 1 ? a_scale : a_gate;
    if constexpr (RB > 1) {
      for (int w = 0; w < RB; ++w) {
        __syncthreads();
        if (rb == w) {
#pragma unroll
          for (int i = 0; i < GP; ++i) {
            if (!has[i]) continue;
            float* at = vec + (t + i * T) * 4;
#pragma unroll
            for (int e = 0; e < 8; ++e) at[at_vec(0, e)] = w == 0 ? a[i][e] : at[at_vec(0, e)] + a[i][e];
          }
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < p.C; c += NT) out[q * p.C + c] = vec[at_vec(c / 8, c % 8)];
    } else {
#pragma unroll
      for (int i = 0; i < GP; ++i) {
        if (!has[i]) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) out[q * p.C + (t + i * T) * 8 + e] = a[i][e];
      }
    }
  }
}

// The gradients shared between rows from the chunks' sums: 6 to 10 us, latency of
// three dependent loads and a launch.  Work-group (x, y):
// 64 columns, a wave per 16th of the chunks; y < B G: shift, scale and gate of a
// batch entry and group; the last y: the weights, over all of them.
__global__ __launch_bounds__(1024) void norm_shared_kernel(const NormParams p) {
  __shared__ float part[16][3][64];
  const int lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool in = c < p.C;
  const auto bf = [&](const uint16_t* v, int64_t at) { return __uint_as_float(uint32_t(v[at]) << 16); };
  const int one = int(blockIdx.y), all = p.B * p.G;
  float sum[3] = {0.f, 0.f, 0.f};
  // a 16th of the flat list (batch entry, chunk) of a batch entry, or of all, in
  // runs inside one span, eight chunks' loads in flight
  const int first = one < all ? one / p.G * p.chunks : 0, n = one < all ? p.chunks : p.B * p.chunks;
  const int last = first + int(int64_t(n) * (wave + 1) / 16);
  for (int k = first + int(int64_t(n) * wave / 16); k < last;) {
    const int b = k / p.chunks, chunk = k - b * p.chunks;
    int s = 0;
    while (s + 1 < p.n_spans && p.span_chunk0[s + 1] <= chunk) ++s;
    const int g = p.span_group[s];
    const int stop = min(last, b * p.chunks + (s + 1 < p.n_spans ? p.span_chunk0[s + 1] : p.chunks));
    if (in && (one == all || g == one % p.G)) {
      float a[3] = {0.f, 0.f, 0.f};
      const float* q = p.partial + int64_t(k) * 3 * p.C + c;
      for (int m = stop - k; m > 0; m -= 8, q += int64_t(8) * 3 * p.C) {
        float v[8][3];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 3; ++i) v[j][i] = j < m ? q[int64_t(j * 3 + i) * p.C] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 3; ++i) a[i] += v[j][i];
      }
      if (one == all) {
        const int64_t mod = b * p.mod_sb + int64_t(g) * p.mod_sg + c;
        if (p.scale) a[1] *= 1.f + bf(p.scale, mod);
        if (p.gate) a[2] *= bf(p.gate, mod);
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) sum[i] += a[i];
    }
    k = stop;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) part[wave][i][lane] = sum[i];
  __syncthreads();
  if (wave > 2 || !in) return;  // a wave per sum
  float x = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) x += part[w][wave][lane];
  const int64_t at = int64_t(one) * p.C + c;
  if (one == all) {
    if (wave == 1 && p.dweight) p.dweight[c] = x;
    if (wave == 2 && p.dpost_weight) p.dpost_weight[c] = x;
    return;
  }
  if (wave == 0 && p.dshift) p.dshift[at] = x;
  if (wave == 1 && p.dscale) p.dscale[at] = x * (p.weight ? bf(p.weight, c) : 1.f);
  if (wave == 2 && p.dgate) p.dgate[at] = x * (p.post_weight ? bf(p.post_weight, c) : 1.f);
}

template <int T, int GP>
void launch_fwd(const NormParams& p, hipStream_t s) {
  const int64_t rows = p.N * p.B;
  hipLaunchKernelGGL((norm_kernel<T, GP>), dim3((rows + 256 / T - 1) / (256 / T)), dim3(256), 0, s, p);
}
template <int T, int GP>
void launch_bwd(const NormParams& p, hipStream_t s) {
  if (p.chunks > 0)
    hipLaunchKernelGGL((norm_backward_kernel<T, GP>), dim3(int64_t(p.B) * p.chunks), dim3(512), 0, s, p);
  const int weights = p.dweight || p.dpost_weight, vectors = p.dshift || p.dscale || p.dgate;
  if (weights || vectors)
    hipLaunchKernelGGL(norm_shared_kernel, dim3((p.C + 63) / 64, p.B * p.G + weights), dim3(1024), 0, s, p);
}

}  // namespace

// Threads per row and granules per thread, by the row's granules.  A row inside
// one wave needs no barrier; with more than two or three granules a thread the
// registers leave too few waves and loads.  21 M values, us with 64, 128 and 256
// threads a row (one set of rows again and again):
//   C           512    1024    1928    2560    4096
//   forward    28.6    26.9    30.4    26.8    33.3
//              33.5    28.7    28.1    25.6    26.4
//              46.1    32.7    29.7    26.1    26.5
//   backward   56.4    57.4    64.4   125.6       -
//              88.9    65.5    66.1    65.3    67.2
//             156.2    91.1    71.0    68.5    64.4
// Backward, 1032 to 2048 channels: 64 threads, 128 here, are better for many rows and
// worse for few (new rows each call: 10877 rows of 1928 63.9 with 64, 65.8 with 128, 10877
// of 1160 46.0 and 52.2, two samples' 3936 of 1928 55.1 and 57.6; but 1417 rows of 2048
// 27.1 and 23.7, 80 rows 21.5 and 17.9).  128 lose at most 14%, 64 up to 20%.
int launch_norm(const NormParams& p, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int ng = p.C / 8;
  if (ng <= 64) launch_fwd<64, 1>(p, s);
  else if (ng <= 128) launch_fwd<64, 2>(p, s);
  else if (ng <= 256) launch_fwd<128, 2>(p, s);
  else if (ng <= 384) launch_fwd<128, 3>(p, s);
  else if (ng <= 512) launch_fwd<256, 2>(p, s);
  else if (ng <= 1024) launch_fwd<256, 4>(p, s);
  else launch_fwd<256, 8>(p, s);
  return int(hipGetLastError());
}

int launch_norm_backward(const NormParams& p, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int ng = p.C / 8;
  if (ng <= 64) launch_bwd<64, 1>(p, s);
  else if (ng <= 128) launch_bwd<64, 2>(p, s);
  else if (ng <= 256) launch_bwd<128, 2>(p, s);
  else if (ng <= 384) launch_bwd<128, 3>(p, s);
  else if (ng <= 512) launch_bwd<256, 2>(p, s);
  else if (ng <= 1024) launch_bwd<512, 2>(p, s);
  else launch_bwd<512, 4>(p, s);
  return int(hipGetLastError());
}

}  // namespace rc
