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
  int32_t piece0;     // first piece, over the segments of both kinds in launch order, per (batch, head)
  int32_t r0, nr;     // streamed ranges
  int32_t keys;       // own rows are keys
  int32_t splits;     // pieces of a tile's streamed rows; > 1: fp32 partials, merged by a second launch
  int32_t slot0;      // first partial, per (batch, head), in units of one output's own x D
};
struct BwdRange {
  int32_t start, len;
};

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
  float* partial;      // [slots B H, own, D] in accumulator order
  int32_t own;         // own rows of a tile: 256, or 128
  int32_t n_seg, n_pieces, n_slots;
  BwdSeg seg[2 * RC_MAX_SEGMENTS];
  BwdRange range[2 * kMaxRanges];
};
int launch_attention_bwd(const BwdParams& p, int D, void* stream) RC_WEAK;

// ---------------------------------------------------------------- rotation
struct RotaryParams {
  const uint16_t* x[2];   // queries, keys (null: none); backward: the gradients of the outputs
  const uint16_t* n[2];   // backward with a norm: its inputs
  uint16_t* y[2];
  const uint16_t* w[2];   // norm weights [D], null: no norm
  float* dw[2];           // backward: their gradients
  float* partial;         // backward: [blocks, 2, D] sums of dw
  const void* pos;        // [N, axes] or [B, N, axes], int32 or fp32
  int64_t x_st, n_st, y_st, pos_sb;
  int64_t N;
  int32_t B, H, axes, pos_float;
  int32_t groups;         // row groups (64 lanes of 16 bytes each) per wave
  int32_t blocks;         // backward with a norm: work-groups of the first pass
  float eps, sign;        // sign: -1 turns back
  int32_t width;          // rotated channels, the first ones of a head row
  int32_t half;           // > 0: channel p pairs with p + half; 0: 2p with 2p + 1
  uint8_t axis[64];
  double turns[64];       // per pair, revolutions per unit of position; 0 past the rotated width
};
int launch_rotary(const RotaryParams& p, int D, void* stream) RC_WEAK;
int launch_rotary_norm_backward(const RotaryParams& p, int D, void* stream) RC_WEAK;
constexpr int kRotaryBlocks = 768;  // work-groups of the backward with a norm, at most (three per CU)

// ---------------------------------------------------------------- gated norm
struct NormRows {  // [B * N, C] rows
  uint16_t* p;
  int64_t ld;
};
struct NormParams {
  NormRows h, x, h_out, y;            // forward
  NormRows dy, dh, dh_in, dx;         // backward (h: the rows after the residual)
  const uint16_t *gate, *scale, *shift, *weight, *post_weight;
  float *dgate, *dscale, *dshift, *dweight, *dpost_weight;
  float* partial;                     // [B, chunks, 3, C]
  int64_t mod_sb, mod_sg;             // element strides of gate, scale and shift
  int64_t N;
  int32_t B, C, G, rms, post;
  float eps, rscale, inv_c;
  int32_t n_spans;
  int32_t chunk_rows, chunks;         // backward: rows of a chunk (inside one span), chunks per batch entry
  int32_t span_row0[RC_MAX_SEGMENTS], span_rows[RC_MAX_SEGMENTS], span_group[RC_MAX_SEGMENTS];
  int32_t span_chunk0[RC_MAX_SEGMENTS];
};
constexpr int kNormMaxC = 16384;
int launch_norm(const NormParams& p, void* stream) RC_WEAK;
int launch_norm_backward(const NormParams& p, void* stream) RC_WEAK;

}  // namespace rc
