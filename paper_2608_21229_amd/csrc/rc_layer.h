// Internal declarations of the layer operators around the attention: the
// gradient of the full recompute, the rotation of queries and keys, the gated
// norm.  Not part of the public ABI.
#pragma once
#include <stdint.h>

#include "rc_internal.h"

// The host planner also builds without the kernels (its sanitizer build), so
// the launchers of these operators are weak there: a null one is an error.
#define RC_WEAK __attribute__((weak))

namespace rc {

// ---------------------------------------------------------------- attention gradient
// Two kinds of work-groups pass over the visible (query, key) pairs: those that
// hold queries sum dQ, those that hold keys sum dK and dV.  The rows a
// work-group holds are its own, the rows they meet are streamed.
struct BwdSeg {
  int32_t row0, len;  // own rows
  int32_t tile0;      // first own tile, over the segments of both kinds in launch order
  int32_t r0, nr;     // streamed ranges
  int32_t keys;       // own rows are keys
};
struct BwdRange {
  int32_t start, len;
};
constexpr int kBwdOwn = 256;  // own rows of a tile

struct BwdParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* o;
  const uint16_t* d_o;
  const float* lse;
  const float* dlse;   // null: none
  uint16_t* dq;
  uint16_t* dk;
  uint16_t* dv;
  float* nlse;         // [B, H, N] -lse / scale
  float* ndelta;       // [B, H, N] dlse - sum_d dO O
  int64_t st, g_st;    // token strides (elements) of Q/K/V and of the gradients; batch stride N times that
  int32_t B, H, n_rows;
  float scale, scale_log2;
  int32_t n_seg, n_tiles;
  BwdSeg seg[2 * RC_MAX_SEGMENTS];
  BwdRange range[2 * kMaxRanges];
};
int launch_attention_bwd(const BwdParams& p, int D, void* stream) RC_WEAK;

}  // namespace rc
