// Stand-ins for the kernel launchers of the 8-bit projections, linked with the
// host planner and stub_launchers.cpp.  Each checks what it is handed and aborts
// on a broken invariant; the last call's figures are there for the cases.
#include <stdio.h>
#include <stdlib.h>

#include "rc_blocks8.h"

namespace {

long g_launches = 0, g_tile = -1, g_splits = 0, g_whole = 0, g_few = 0;
const uint8_t* g_lo = nullptr;  // workspace range that a call may write
const uint8_t* g_hi = nullptr;

[[noreturn]] void fail(const char* what, long a, long b) {
  fprintf(stderr, "stub launcher: broken call: %s (%ld, %ld)\n", what, a, b);
  fflush(stderr);
  abort();
}
#define REQUIRE(cond, a, b) \
  do {                      \
    if (!(cond)) fail(#cond, long(a), long(b)); \
  } while (0)

void check_blocks(const rc::Blocks8& b, int64_t rows, int64_t cols) {
  REQUIRE(b.codes && b.exps && (uintptr_t(b.codes) & 15) == 0 && (uintptr_t(b.exps) & 15) == 0, rows, cols);
  REQUIRE(b.ld >= rc::pad8(cols) && b.ld % 16 == 0 && b.ld <= rc::kMaxCols8, b.ld, cols);
  REQUIRE(b.le >= rows && b.le % 16 == 0 && b.le <= rc::kMaxRows8, b.le, rows);
}

void check_inside(const void* p, int64_t bytes) {
  const uint8_t* q = static_cast<const uint8_t*>(p);
  REQUIRE(q >= g_lo && q + bytes <= g_hi, bytes, g_hi - g_lo);
}

}  // namespace

namespace rc {

int launch_quantize_rows(const Quant8Params& q, void*) {
  REQUIRE(q.x && q.ldx >= q.K && q.M >= 1 && q.K % 8 == 0 && !q.out_t.codes, q.M, q.K);
  check_blocks(q.out, q.M, q.K);
  if (g_lo && q.out.codes >= g_lo && q.out.codes < g_hi) {
    check_inside(q.out.codes, q.M * q.out.ld);
    check_inside(q.out.exps, blocks8(q.K) * q.out.le);
  }
  ++g_launches;
  return 0;
}

int launch_quantize_squares(const Quant8Params& q, void*) {
  REQUIRE(q.x && q.ldx >= q.K && q.M >= 1 && q.K % 8 == 0, q.M, q.K);
  check_blocks(q.out, q.M, q.K);
  if (q.out_t.codes) check_blocks(q.out_t, q.K, q.M);
  ++g_launches;
  return 0;
}

int launch_dequantize(const Dequant8Params& q, void*) {
  REQUIRE(q.out && q.ldo >= q.K && q.M >= 1, q.M, q.K);
  check_blocks(q.x, q.M, q.K);
  ++g_launches;
  return 0;
}

int launch_linear8(const Linear8Params& q, int32_t tile, void*) {
  REQUIRE(tile >= 0 && tile < int(sizeof kLinear8Tiles / sizeof *kLinear8Tiles), tile, 0);
  REQUIRE(q.out && q.ldo >= q.N && (!q.r || q.ldr >= q.N) && q.M >= 1, q.M, q.N);
  check_blocks(q.a, q.M, q.K);
  check_blocks(q.w, q.N, q.K);
  REQUIRE((q.M + kLinear8Tiles[tile].bm - 1) / kLinear8Tiles[tile].bm * ((q.N + 63) / 64) < int64_t(1) << 31, q.M, q.N);
  g_tile = tile;
  g_few = 0;
  ++g_launches;
  return 0;
}

int launch_linear8_few(const Linear8Params& q, void*) {
  REQUIRE(q.x && q.ldx >= q.K && q.out && q.ldo >= q.N && (!q.r || q.ldr >= q.N) && q.M >= 1, q.M, q.N);
  REQUIRE((q.M + 15) / 16 <= 65535, q.M, 0);  // rows of the grid
  check_blocks(q.w, q.N, q.K);
  g_few = 1;
  ++g_launches;
  return 0;
}

int launch_wgrad8(const WGrad8Params& q, int32_t tile, void*) {
  REQUIRE(tile >= 0 && tile < int(sizeof kWGrad8Tiles / sizeof *kWGrad8Tiles), tile, 0);
  REQUIRE(q.dw && q.lddw >= q.K && q.M >= 0, q.M, q.K);
  if (q.M > 0) {
    REQUIRE(q.dy && q.lddy >= q.N, q.lddy, q.N);
    check_blocks(q.x, q.M, q.K);
  }
  const Tile8 t = kWGrad8Tiles[tile];
  const int64_t tiles = int64_t((q.N + t.bm - 1) / t.bm) * ((q.K + t.bn - 1) / t.bn), rest = tiles - q.whole;
  REQUIRE(q.whole >= 0 && q.whole % kCUs == 0 && rest >= 0 && rest < kCUs, q.whole, tiles);
  REQUIRE(q.splits >= 1 && rest * q.splits <= kCUs, q.splits, rest);
  REQUIRE(q.splits == 1 || (rest > 0 && q.splits <= (q.M + 63) / 64), q.splits, q.M);
  if (q.splits > 1) {
    REQUIRE((uintptr_t(q.partial) & 15) == 0, 0, 0);
    if (g_lo) check_inside(q.partial, rest * q.splits * t.bm * t.bn * 4);
  }
  g_tile = tile;
  g_splits = q.splits;
  g_whole = q.whole;
  ++g_launches;
  return 0;
}

}  // namespace rc

extern "C" {
long rc_stub_blocks8_launches() { return g_launches; }
long rc_stub_blocks8_tile() { return g_tile; }
long rc_stub_blocks8_splits() { return g_splits; }
long rc_stub_blocks8_whole() { return g_whole; }
long rc_stub_blocks8_few() { return g_few; }
long rc_stub_blocks8_workspace(uintptr_t at, long bytes) {
  g_lo = reinterpret_cast<const uint8_t*>(at);
  g_hi = g_lo + bytes;
  return 0;
}
}
