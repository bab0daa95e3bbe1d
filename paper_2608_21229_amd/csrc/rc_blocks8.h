// Internal declarations of the projections in 8 bits: e4m3 codes with one
// power-of-two scale per block of 128 values, their product, and the gradient
// of the weights from an 8-bit checkpoint.  Not part of the public ABI.
#pragma once
#include <stdint.h>

#include "rc_internal.h"

// As the layer operators': the host planner also builds without the kernels.
#ifndef RC_WEAK
#define RC_WEAK __attribute__((weak))
#endif

namespace rc {

constexpr int kBlock8 = 128;                      // values that share a scale
constexpr int64_t kMaxRows8 = int64_t(1) << 28;   // a tile's scales are addressed with 32-bit offsets
constexpr int32_t kMaxCols8 = 1 << 22;            // and so are a tile's rows

constexpr int64_t blocks8(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }
constexpr int64_t pad8(int64_t n) { return blocks8(n) * kBlock8; }
constexpr int64_t pitch8(int64_t rows) { return (rows + 15) / 16 * 16; }

// codes[row * ld + col], exponent + 127 of the block of (row, col) at exps[col / 128 * le + row].
struct Blocks8 {
  uint8_t* codes;
  int64_t ld;
  uint8_t* exps;
  int64_t le;
};

struct Quant8Params {
  const uint16_t* x;
  int64_t ldx;
  int64_t M;
  int32_t K;
  Blocks8 out, out_t;  // out_t.codes null: not transposed
};
int launch_quantize_rows(const Quant8Params& q, void* stream) RC_WEAK;
int launch_quantize_squares(const Quant8Params& q, void* stream) RC_WEAK;

struct Dequant8Params {
  Blocks8 x;
  int64_t M;
  int32_t K;
  uint16_t* out;
  int64_t ldo;
};
int launch_dequantize(const Dequant8Params& q, void* stream) RC_WEAK;

struct Linear8Params {
  const uint16_t* x;   // few rows: bf16 [M, K], quantised on the way; else null
  int64_t ldx;
  Blocks8 a, w;        // [M, K] and [N, K]
  const uint16_t* r;   // [M, N] or null
  uint16_t* out;       // [M, N]
  int64_t M, ldr, ldo;
  int32_t N, K;
};
int launch_linear8(const Linear8Params& q, int32_t tile, void* stream) RC_WEAK;
int launch_linear8_few(const Linear8Params& q, void* stream) RC_WEAK;

struct WGrad8Params {
  const uint16_t* dy;  // [M, N]
  int64_t lddy;
  Blocks8 x;           // [M, K]
  float* dw;           // [N, K]
  int64_t lddw;
  float* partial;      // [splits, other tiles][tile]; splits > 1
  int64_t M;
  int32_t N, K;
  int64_t whole;       // tiles that one work-group computes
  int32_t splits;      // work-groups that share the rows of each other tile
};
int launch_wgrad8(const WGrad8Params& q, int32_t tile, void* stream) RC_WEAK;

// Products that quantise their bf16 rows themselves, in one launch: up to 32 rows
// (2 x 7680 x 2560 6.6 us, 32 rows 11.4; the quantisation's launch and the product's
// 4 + 9.5 and the host's time for a second launch), or little to read for each
// group of 32 rows (80 x 384 x 128 3.6 us, as much as the quantisation alone).
constexpr int64_t kFewRows8 = 32, kFewRead8 = int64_t(4) << 20;
constexpr bool few_rows8(int64_t M, int32_t N, int32_t K) {
  return M <= kFewRows8 || (M + 31) / 32 <= kFewRead8 / (N * pad8(K));
}

struct Tile8 {
  int32_t bm, bn;
};
constexpr Tile8 kLinear8Tiles[] = {{256, 256}, {192, 256}, {256, 128}, {128, 128}, {64, 128}, {64, 64}};
int32_t plan_linear8(int64_t M, int32_t N, int32_t K);

// n x k
constexpr Tile8 kWGrad8Tiles[] = {{256, 256}, {256, 128}, {128, 128}};
struct WGrad8Plan {
  int32_t tile, splits;
  int64_t whole, tiles;
  int64_t blocks() const { return whole + (tiles - whole) * splits; }
  size_t partial_bytes() const {
    return splits > 1 ? size_t(blocks() - whole) * kWGrad8Tiles[tile].bm * kWGrad8Tiles[tile].bn * sizeof(float) : 0;
  }
};
WGrad8Plan plan_wgrad8(int64_t M, int32_t N, int32_t K);

}  // namespace rc
