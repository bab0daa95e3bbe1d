// Stand-ins for the layer operators' kernel launchers (attention gradient,
// rotation, gated norm), linked with the host planner and stub_launchers.cpp.
// Each checks the schedule it is handed and aborts on a broken invariant.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include "rc_layer.h"

namespace {

long g_pieces = 0, g_slots = 0, g_own = 0, g_chunks = 0, g_launches = 0;
long g_pairs[2] = {0, 0};

[[noreturn]] void fail(const char* what, long a, long b) {
  fprintf(stderr, "stub launcher: broken schedule: %s (%ld, %ld)\n", what, a, b);
  fflush(stderr);
  abort();
}
#define REQUIRE(cond, a, b) \
  do {                      \
    if (!(cond)) fail(#cond, long(a), long(b)); \
  } while (0)

}  // namespace

namespace rc {

int launch_attention_bwd(const BwdParams& p, int D, void*) {
  REQUIRE(D == 64 || D == 128, D, 0);
  REQUIRE(p.own == 128 || p.own == 256, p.own, 0);
  REQUIRE(p.n_seg >= 1 && p.n_seg <= 2 * RC_MAX_SEGMENTS, p.n_seg, 0);
  REQUIRE(p.q && p.k && p.v && p.o && p.d_o && p.lse && p.dq && p.dk && p.dv && p.nlse && p.ndelta && p.partial, 0, 0);
  REQUIRE(isfinite(p.scale) && p.scale > 0 && fabsf(p.scale_log2 - p.scale * 1.44269504f) <= 1e-6f * p.scale_log2, 0, 0);
  REQUIRE(p.ndelta - p.nlse >= int64_t(p.B) * p.H * p.n_rows, 0, 0);
  REQUIRE(p.partial - p.ndelta >= int64_t(p.B) * p.H * p.n_rows, 0, 0);
  long pieces = 0, slots = 0;
  long rows[2] = {0, 0};
  g_pairs[0] = g_pairs[1] = 0;
  char* seen[2] = {static_cast<char*>(calloc(size_t(p.n_rows), 1)), static_cast<char*>(calloc(size_t(p.n_rows), 1))};
  for (int i = 0; i < p.n_seg; ++i) {
    const BwdSeg& s = p.seg[i];
    REQUIRE(s.len >= 1 && s.row0 >= 0 && int64_t(s.row0) + s.len <= p.n_rows, i, s.row0);
    REQUIRE(s.keys == 0 || s.keys == 1, i, s.keys);
    REQUIRE(s.splits >= 1, i, s.splits);
    REQUIRE(s.piece0 == pieces && s.slot0 == slots, s.piece0, s.slot0);
    REQUIRE(s.nr >= 0 && s.r0 >= s.keys * kMaxRanges && s.r0 + s.nr <= (s.keys + 1) * kMaxRanges, s.r0, s.nr);
    const int own = (s.len + p.own - 1) / p.own;
    long tiles = 0, end = 0;
    for (int r = 0; r < s.nr; ++r) {
      const BwdRange& g = p.range[s.r0 + r];
      REQUIRE(g.len >= 1 && g.start >= end && int64_t(g.start) + g.len <= p.n_rows, r, g.start);
      REQUIRE(r == 0 || g.start > end, r, g.start);  // adjacent ranges are merged
      end = g.start + g.len;
      tiles += (g.len + 63) / 64;
      g_pairs[s.keys] += long(s.len) * g.len;
    }
    REQUIRE(s.splits == 1 || tiles / s.splits >= 1, tiles, s.splits);  // no empty piece
    pieces += long(own) * s.splits;
    if (s.splits > 1) slots += long(own) * s.splits * (1 + s.keys);
    for (int r = 0; r < s.len; ++r) {
      REQUIRE(!seen[s.keys][s.row0 + r], s.keys, s.row0 + r);
      seen[s.keys][s.row0 + r] = 1;
    }
    rows[s.keys] += s.len;
  }
  free(seen[0]);
  free(seen[1]);
  REQUIRE(rows[0] == p.n_rows && rows[1] == p.n_rows, rows[0], rows[1]);
  REQUIRE(pieces == p.n_pieces && slots == p.n_slots, p.n_pieces, p.n_slots);
  REQUIRE(g_pairs[0] == g_pairs[1], g_pairs[0], g_pairs[1]);
  g_pieces = pieces;
  g_slots = slots;
  g_own = p.own;
  ++g_launches;
  return 0;
}

static void check_rotary(const RotaryParams& p, int D) {
  REQUIRE(D == 64 || D == 128, D, 0);
  REQUIRE(p.x[0] || p.x[1], 0, 0);
  REQUIRE(p.N >= 1 && p.B >= 1 && p.H >= 1 && p.axes >= 1, p.N, p.H);
  REQUIRE(p.half % 8 == 0 && p.half * 2 <= D, p.half, D);
  for (int k = 0; k < 2; ++k) {
    REQUIRE(!p.x[k] || p.y[k], k, 0);
    REQUIRE(!p.w[k] || p.x[k], k, 0);
  }
  for (int i = 0; i < 64; ++i) REQUIRE(p.axis[i] < p.axes && isfinite(p.turns[i]), i, p.axis[i]);
}
int launch_rotary(const RotaryParams& p, int D, void*) {
  check_rotary(p, D);
  REQUIRE(p.groups >= 1, p.groups, 0);
  ++g_launches;
  return 0;
}
int launch_rotary_norm_backward(const RotaryParams& p, int D, void*) {
  check_rotary(p, D);
  REQUIRE(p.blocks >= 1 && p.blocks <= kRotaryBlocks && p.partial, p.blocks, 0);
  for (int k = 0; k < 2; ++k) REQUIRE(!p.w[k] || p.n[k], k, 0);
  ++g_launches;
  return 0;
}

int launch_norm(const NormParams& p, void*) {
  REQUIRE(p.C % 8 == 0 && p.C <= kNormMaxC && p.h.p && (p.y.p || p.x.p), p.C, 0);
  REQUIRE((p.x.p == nullptr) == (p.h_out.p == nullptr), 0, 0);
  ++g_launches;
  return 0;
}
int launch_norm_backward(const NormParams& p, void*) {
  int64_t rows = 0, chunks = 0;
  for (int s = 0; s < p.n_spans; ++s) {
    REQUIRE(p.span_rows[s] >= 1 && p.span_row0[s] == rows && p.span_group[s] >= 0 && p.span_group[s] < p.G, s, rows);
    REQUIRE(p.span_chunk0[s] == chunks, s, chunks);
    rows += p.span_rows[s];
    chunks += (p.span_rows[s] + p.chunk_rows - 1) / p.chunk_rows;
  }
  REQUIRE(rows == p.N && chunks == p.chunks, rows, chunks);
  REQUIRE(chunks * p.B <= (p.n_spans * p.B > kCUs ? int64_t(p.n_spans) * p.B : kCUs), chunks, p.B);
  REQUIRE(p.chunks == 0 || p.partial, 0, 0);
  g_chunks = long(chunks);
  ++g_launches;
  return 0;
}

}  // namespace rc

extern "C" {
long rc_stub_layer_launches() { return g_launches; }
long rc_stub_layer_pieces() { return g_pieces; }
long rc_stub_layer_slots() { return g_slots; }
long rc_stub_layer_own() { return g_own; }
long rc_stub_layer_pairs(int keys) { return g_pairs[keys]; }
long rc_stub_layer_chunks() { return g_chunks; }
}
