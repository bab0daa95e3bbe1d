// extern "C" entry points of librefcache: argument validation, planning and
// kernel launches.  Every check runs before the first HIP call, so a failing
// call launches nothing and needs no GPU.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "rc_layer.h"

namespace rc {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

rc_status check_dims(int32_t B, int32_t H, int32_t D, float scale) {
  if (B < 1 || H < 1 || B > 65535 || H > 65535) {
    set_error("B = %d, H = %d: each must be in [1, 65535]", B, H);
    return RC_ERR_ARG;
  }
  if (D != 64 && D != 128) {
    set_error("head_dim %d is not supported (64 or 128)", D);
    return RC_ERR_UNSUPPORTED;
  }
  if (!(scale > 0.f) || !isfinite(scale)) {
    set_error("softmax scale must be finite and > 0 (got %g)", (double)scale);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

rc_status check_ptr(const void* p, const char* name) {
  if (!p) {
    set_error("%s is null", name);
    return RC_ERR_ARG;
  }
  if (!aligned16(p)) {
    set_error("%s is not 16-byte aligned", name);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

rc_status check_lse(const float* p, const char* name) {
  if (p && (reinterpret_cast<uintptr_t>(p) & 3u)) {
    set_error("%s is not 4-byte aligned", name);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

rc_status check_stride(int64_t tok_stride, int32_t H, int32_t D) {
  if (tok_stride < int64_t(H) * D || (tok_stride & 7)) {
    set_error("tok_stride %lld must be >= H*D = %d and a multiple of 8", (long long)tok_stride, H * D);
    return RC_ERR_ARG;
  }
  // a 64-token tile of the source spans 128 * tok_stride bytes, addressed
  // with 32-bit buffer offsets
  if (tok_stride > (int64_t(1) << 24)) {
    set_error("tok_stride %lld is too large (at most 2^24 elements)", (long long)tok_stride);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

rc_status check_blocks(int64_t blocks, const char* what) {
  if (blocks >= (int64_t(1) << 31)) {
    set_error("%s launch of %lld work-groups exceeds the grid limit", what, (long long)blocks);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

rc_status check_grid(const Params& p) {
  return check_blocks(int64_t(p.B) * p.H * p.n_qtiles * p.splits, "attention");
}

#define RC_TRY(x)                  \
  do {                             \
    rc_status _s = (x);            \
    if (_s != RC_OK) return _s;    \
  } while (0)

rc_status hip_status(int err, const char* what) {
  if (err != 0) {
    set_error("%s: HIP error %d", what, err);
    return RC_ERR_HIP;
  }
  return RC_OK;
}

size_t balanced_workspace_bytes(int32_t D) {
  return size_t(2) * kBalancedWGs * rows_per_wg(kQBBalanced) * size_t(D + 2) * sizeof(float);
}

// A bf16 key source from element strides (batch, head, token) shared by K and V.
KeySrc bf16_source(const void* k, const void* v, int64_t sb, int64_t sh, int64_t st) {
  return KeySrc{static_cast<const char*>(k), static_cast<const char*>(v), 2 * sb, 2 * sh, 2 * st, 2 * sb, 2 * sh,
                2 * st};
}

void fill_common(Params& p, int32_t B, int32_t H, float scale) {
  p.B = B;
  p.H = H;
  p.splits = 1;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.lse = nullptr;
  p.ws_o = nullptr;
  p.ws_ml = nullptr;
  p.src[1] = KeySrc{nullptr, nullptr, 0, 0, 0, 0, 0, 0};
}

}  // namespace
}  // namespace rc

namespace rc {
namespace {

// The prefill's schedule: query tiles and key ranges, the copy work-groups
// (amax work-groups for the FP8 cache) and the cache rows they take, in p
// (p.B and p.H set by the caller).
rc_status plan_prefill(const rc_layout* L, int32_t D, bool fp8, Params& p) {
  p.bm = rows_per_wg(kQBPlain);
  RC_TRY(plan(L, RC_ENTRY_PREFILL, p));
  const int64_t n_cached = count_cached_rows(L);
  const CopyPlan c = fp8 ? plan_amax_tail(p, n_cached, D) : plan_copy_tail(p, n_cached);
  p.cp.blocks = c.blocks;
  p.cp.rows = int32_t(c.rows);
  p.half_tiles = half_tiles(p);
  return RC_OK;
}

// The full recompute's schedule; last_round: with the workspace that lets it
// split the grid's partial last round.
rc_status plan_full(const rc_layout* L, bool last_round, Params& p) {
  p.bm = rows_per_wg(kQBPlain);
  RC_TRY(plan(L, RC_ENTRY_FULL, p));
  if (last_round) p.lr_tiles = last_round_tiles(p);
  p.splits = p.lr_tiles > 0 ? 2 : 1;
  if (p.lr_tiles == 0) p.tail_num = 0;
  p.half_tiles = half_tiles(p);
  return RC_OK;
}

// The prefill of both cache formats: static-row attention, then the bf16 cache
// store or the FP8 quantising store.
rc_status prefill_impl(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale, const void* q_static,
                       const void* k_static, const void* v_static, int64_t tok_stride, void* o_static,
                       float* lse_static, bool fp8, void* k_cache, void* v_cache, float* kv_scale, void* stream) {
  RC_TRY(check_layout(L, RC_ENTRY_PREFILL));
  RC_TRY(check_dims(B, H, D, scale));
  RC_TRY(check_stride(tok_stride, H, D));
  const int64_t n_static = count_rows(L, RowSet::Static);
  const int64_t n_cached = count_cached_rows(L);
  if (n_static == 0) return RC_OK;  // no ST/R segment: nothing to prefill
  RC_TRY(check_ptr(q_static, "q_static"));
  RC_TRY(check_ptr(k_static, "k_static"));
  RC_TRY(check_ptr(v_static, "v_static"));
  RC_TRY(check_ptr(o_static, "o_static"));
  RC_TRY(check_lse(lse_static, "lse_static"));
  if (fp8) {
    // the scales are required whatever the cache size, so that a caller's
    // missing buffer is caught here rather than on the device
    if (!kv_scale) {
      set_error("kv_scale is null");
      return RC_ERR_ARG;
    }
    RC_TRY(check_lse(kv_scale, "kv_scale"));
  }
  if (n_cached > 0) {
    RC_TRY(check_ptr(k_cache, fp8 ? "k_cache8" : "k_cache"));
    RC_TRY(check_ptr(v_cache, fp8 ? "v_cache8" : "v_cache"));
    if (fp8 && n_cached > kFp8MaxKeys) {
      set_error("FP8 cache of %lld keys per (batch, head) exceeds %lld", (long long)n_cached,
                (long long)kFp8MaxKeys);
      return RC_ERR_ARG;
    }
  }
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, scale);
  RC_TRY(plan_prefill(L, D, fp8, p));
  RC_TRY(check_grid(p));
  p.q = static_cast<const uint16_t*>(q_static);
  p.q_st = tok_stride;
  p.q_sb = tok_stride * n_static;
  p.o = static_cast<uint16_t*>(o_static);
  p.o_st = int64_t(H) * D;
  p.o_sb = p.o_st * n_static;
  p.lse = lse_static;
  p.src[0] = bf16_source(k_static, v_static, tok_stride * n_static, D, tok_stride);

  // the cached segments' rows inside the static buffers and their cache
  // positions; segments that follow each other in both are one run, since the
  // copy and amax loops walk the whole run table for every row (FP8 prefill of
  // 8 heads, D = 128, paper mask: 20 references of 512 tokens 547 us in 20
  // runs, 419 in one; of 128 tokens 142 and 84)
  CopySeg seg[RC_MAX_SEGMENTS];
  int n_copy = 0;
  {
    const uint32_t cm = cached_mask(L);
    int32_t srow = 0, drow = 0;
    for (int i = 0; i < L->n_seg; ++i) {
      if (!is_static_kind(L->seg[i].kind)) continue;
      if (cm >> i & 1u) {
        if (n_copy > 0 && seg[n_copy - 1].src_row0 + seg[n_copy - 1].len == srow) seg[n_copy - 1].len += L->seg[i].len;
        else seg[n_copy++] = CopySeg{srow, L->seg[i].len, drow};
        drow += L->seg[i].len;
      }
      srow += L->seg[i].len;
    }
  }
  if (!fp8) {
    CacheStoreParams c;
    memset(&c, 0, sizeof c);
    if (n_cached > 0) {
      c.k_src = static_cast<const uint16_t*>(k_static);
      c.v_src = static_cast<const uint16_t*>(v_static);
      c.k_dst = static_cast<uint16_t*>(k_cache);
      c.v_dst = static_cast<uint16_t*>(v_cache);
      c.src_st = tok_stride;
      c.src_sb = tok_stride * n_static;
      c.B = B;
      c.H = H;
      c.D = D;
      c.n_cached = int32_t(n_cached);
      c.n_copy = n_copy;
      for (int i = 0; i < n_copy; ++i) c.seg[i] = seg[i];
      c.total_rows = int32_t(n_cached);
    }
    // Copy work-groups at the end of the attention grid take the cache rows
    // that fit on the CUs its partial last round leaves free; the store
    // kernel (one thread per 16-byte granule, 256 per work-group) the rest.
    CopyTail& t = p.cp;
    if (t.blocks > 0) {
      t.k_src = c.k_src;
      t.v_src = c.v_src;
      t.k_dst = c.k_dst;
      t.v_dst = c.v_dst;
      t.src_sb = c.src_sb;
      t.src_st = c.src_st;
      t.B = B;
      t.H = H;
      t.n_cached = c.n_cached;
      t.n_copy = c.n_copy;
      for (int i = 0; i < n_copy; ++i) t.seg[i] = seg[i];
      RC_TRY(check_blocks(int64_t(B) * H * p.n_qtiles + t.blocks, "prefill attention"));
    }
    c.row0 = t.rows;
    const int64_t rest = int64_t(B) * H * n_cached - t.rows;
    RC_TRY(check_blocks((rest * (D / 8) + 255) / 256, "cache store"));
    RC_TRY(hip_status(launch_attention(p, D, stream), "prefill attention launch"));
    if (rest > 0) RC_TRY(hip_status(launch_cache_store(c, stream), "cache store launch"));
    return RC_OK;
  }
  CacheStore8Params c;
  memset(&c, 0, sizeof c);
  c.k_src = static_cast<const uint16_t*>(k_static);
  c.v_src = static_cast<const uint16_t*>(v_static);
  c.k_dst = static_cast<uint8_t*>(k_cache);
  c.v_dst = static_cast<uint8_t*>(v_cache);
  c.kv_scale = kv_scale;
  c.src_st = tok_stride;
  c.src_sb = tok_stride * n_static;
  c.B = B;
  c.H = H;
  c.D = D;
  c.n_cached = int32_t(n_cached);
  c.n_copy = n_copy;
  for (int i = 0; i < n_copy; ++i) c.seg[i] = seg[i];
  // the quantising store's grids: (B H) x row blocks (amax), one thread per
  // 16-byte granule of K and of V
  if (n_cached > 0) {
    // amax work-groups at the end of the attention grid take the (batch,
    // head)s that fit on the CUs its partial last round leaves free
    CopyTail& t = p.cp;
    c.bh0 = t.rows / c.n_cached;
    t.B = B;
    t.H = H;
    if (c.bh0 > 0) {
      t.k_src = c.k_src;
      t.v_src = c.v_src;
      t.src_sb = c.src_sb;
      t.src_st = c.src_st;
      t.n_cached = c.n_cached;
      t.n_copy = c.n_copy;
      for (int i = 0; i < n_copy; ++i) t.seg[i] = seg[i];
      t.amax = kv_scale;
      RC_TRY(check_blocks(int64_t(B) * H * p.n_qtiles + t.blocks, "prefill attention"));
    } else {
      p.amax_clear = kv_scale;
    }
  }
  RC_TRY(check_blocks(int64_t(B) * H, "FP8 cache store"));
  RC_TRY(check_blocks((int64_t(B) * H * n_cached * (D / 8) + 255) / 256, "FP8 cache store"));
  RC_TRY(hip_status(launch_attention(p, D, stream), "prefill attention launch"));
  if (n_cached > 0) RC_TRY(hip_status(launch_cache_store_fp8(c, stream), "FP8 cache store launch"));
  return RC_OK;
}

// The step's schedule for a split choice (0 = automatic): query tiles, key
// ranges and the resolved split count, in p (p.B and p.H set by the caller).
rc_status plan_step(const rc_layout* L, int32_t D, bool fp8, int32_t splits, Params& p) {
  // the automatic choice is the one rc_step_auto_splits reports (for either
  // cache format)
  if (splits == 0) splits = rc_step_auto_splits(L, p.B, p.H, D);
  const bool balanced = splits == kSplitsBalanced;
  p.bm = rows_per_wg(fp8 ? kQBFp8 : balanced ? kQBBalanced : kQBPlain);
  RC_TRY(plan(L, RC_ENTRY_STEP, p, fp8));
  if (splits == kSplitsTail) {
    p.splits = 2;
    p.tail_num = tail_num(p);
  } else if (splits == kSplitsLastRound) {
    p.lr_tiles = last_round_tiles(p);
    p.splits = p.lr_tiles > 0 ? 2 : 1;
  } else {
    p.splits = splits;
  }
  if (balanced) {
    p.units = int64_t(p.B) * p.H * p.units_bh;
    p.bal_wgs = kBalancedWGs;
    return RC_OK;
  }
  p.half_tiles = half_tiles(p);
  return check_grid(p);
}

// The per-step attention over either cache format (bf16, or FP8: K8 and V8
// with their scales).
rc_status step_impl(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale, const void* q_live,
                    const void* k_live, const void* v_live, int64_t tok_stride, bool fp8, const void* k_cache,
                    const void* v_cache, const float* kv_scale, void* o_live, float* lse_live, int32_t splits,
                    void* workspace, size_t ws_bytes, void* stream) {
  RC_TRY(check_layout(L, RC_ENTRY_STEP));
  RC_TRY(check_dims(B, H, D, scale));
  RC_TRY(check_stride(tok_stride, H, D));
  if (splits < kSplitsLastRound || splits > kMaxSplits) {
    set_error("splits = %d must be RC_SPLITS_LAST_ROUND (-3), RC_SPLITS_TAIL (-2), RC_SPLITS_BALANCED (-1) or in "
              "[0, %d]",
              splits, kMaxSplits);
    return RC_ERR_ARG;
  }
  const int64_t n_live = count_rows(L, RowSet::Live);
  const int64_t n_cached = count_cached_rows(L);
  if (fp8 && splits == kSplitsBalanced) {
    set_error("the balanced schedule is not available with the FP8 cache");
    return RC_ERR_UNSUPPORTED;
  }
  if (fp8) {
    // required whatever the cache size (see the prefill)
    if (!kv_scale) {
      set_error("kv_scale is null");
      return RC_ERR_ARG;
    }
    RC_TRY(check_lse(kv_scale, "kv_scale"));
  }
  if (n_live == 0) return RC_OK;  // no LT/X segment: nothing to attend
  RC_TRY(check_ptr(q_live, "q_live"));
  RC_TRY(check_ptr(k_live, "k_live"));
  RC_TRY(check_ptr(v_live, "v_live"));
  RC_TRY(check_ptr(o_live, "o_live"));
  RC_TRY(check_lse(lse_live, "lse_live"));
  if (n_cached > 0) {
    RC_TRY(check_ptr(k_cache, fp8 ? "k_cache8" : "k_cache"));
    RC_TRY(check_ptr(v_cache, fp8 ? "v_cache8" : "v_cache"));
    if (fp8) {
      if (n_cached > kFp8MaxKeys) {
        set_error("FP8 cache of %lld keys per (batch, head) exceeds %lld", (long long)n_cached,
                  (long long)kFp8MaxKeys);
        return RC_ERR_ARG;
      }
    }
  }
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, scale);
  RC_TRY(plan_step(L, D, fp8, splits, p));
  const bool balanced = p.splits == kSplitsBalanced;
  p.q = static_cast<const uint16_t*>(q_live);
  p.q_st = tok_stride;
  p.q_sb = tok_stride * n_live;
  p.o = static_cast<uint16_t*>(o_live);
  p.o_st = int64_t(H) * D;
  p.o_sb = p.o_st * n_live;
  p.lse = lse_live;
  p.src[0] = bf16_source(k_live, v_live, tok_stride * n_live, D, tok_stride);
  if (fp8) {
    p.fp8 = 1;
    p.kv_scale = kv_scale;
    p.src[1] = KeySrc{static_cast<const char*>(k_cache), static_cast<const char*>(v_cache), int64_t(H) * n_cached * D,
                      n_cached * D, D, int64_t(H) * n_cached * D, n_cached * D, D};
  } else {
    p.src[1] = bf16_source(k_cache, v_cache, int64_t(H) * n_cached * D, n_cached * D, D);
  }
  if (balanced) {
    const size_t need = balanced_workspace_bytes(D);
    if (!workspace || !aligned16(workspace) || ws_bytes < need) {
      set_error("the balanced schedule needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? ws_bytes : size_t(0));
      return RC_ERR_WORKSPACE;
    }
    p.ws_o = static_cast<float*>(workspace);
    p.ws_ml = p.ws_o + size_t(2) * kBalancedWGs * rows_per_wg(kQBBalanced) * D;
    RC_TRY(check_blocks((int64_t(B) * H * n_live * (D / 4) + 255) / 256, "balanced merge"));
    RC_TRY(hip_status(launch_attention_balanced(p, D, stream), "step attention launch"));
    RC_TRY(hip_status(launch_combine_balanced(p, D, stream), "balanced merge launch"));
    return RC_OK;
  }
  CombineParams c;
  memset(&c, 0, sizeof c);
  if (p.splits > 1) {
    const size_t need = rc_step_workspace_bytes(L, B, H, D, splits);
    if (!workspace || !aligned16(workspace) || ws_bytes < need) {
      set_error("split-KV with %d splits needs a 16-byte aligned workspace of %zu bytes (got %zu)", p.splits,
                need, workspace ? ws_bytes : size_t(0));
      return RC_ERR_WORKSPACE;
    }
    p.ws_o = static_cast<float*>(workspace);
    p.ws_ml = p.lr_tiles > 0 ? p.ws_o + size_t(2) * p.lr_tiles * p.bm * D
                             : p.ws_o + size_t(p.splits) * B * H * n_live * D;
    c.ws_o = p.ws_o;
    c.ws_ml = p.ws_ml;
    c.o = p.o;
    c.lse = lse_live;
    c.o_sb = p.o_sb;
    c.o_st = p.o_st;
    c.B = B;
    c.H = H;
    c.D = D;
    c.n_rows = int32_t(n_live);
    c.splits = p.splits;
    for (int i = 0; i < p.n_qseg; ++i) {
      c.seg[c.n_seg++] = CombineParams::Seg{p.qseg[i].row0, p.qseg[i].len, c.n_blocks};
      c.n_blocks += (p.qseg[i].len + 31) / 32;
    }
  }
  // combine: one wave per (up to) 32 rows and 32 columns, four per work-group;
  // fewer than 2^31 by this check and the attention grid's
  if (p.splits > 1) RC_TRY(check_blocks((int64_t(B) * H * n_live * (D / 4) + 255) / 256, "split-KV combine"));
  if (p.lr_tiles > 0) RC_TRY(check_blocks(int64_t(B) * H * p.n_qtiles + p.lr_tiles, "step attention"));
  RC_TRY(hip_status(launch_attention(p, D, stream), "step attention launch"));
  if (p.lr_tiles > 0) RC_TRY(hip_status(launch_combine_last_round(p, D, stream), "last-round merge launch"));
  else if (p.splits > 1) RC_TRY(hip_status(launch_combine(c, stream), "split-KV combine launch"));
  return RC_OK;
}

}  // namespace
}  // namespace rc

namespace rc {
namespace {

// The layer operators' launchers are weak: a build without the kernels (the
// sanitizer build of the planner) refuses the call instead.
template <class F>
rc_status check_launcher(F* f, const char* what) {
  if (f == nullptr) {
    set_error("%s: this build has no kernels", what);
    return RC_ERR_HIP;
  }
  return RC_OK;
}

// The layout whose rows are L's keys: segment k "reads" the segments that read
// it.
rc_layout key_layout(const rc_layout* L) {
  rc_layout t = *L;
  for (int k = 0; k < L->n_seg; ++k) {
    t.visible[k] = 0;
    for (int q = 0; q < L->n_seg; ++q)
      if (L->visible[q] >> k & 1u) t.visible[k] |= 1u << q;
  }
  return t;
}

// Own tiles have 256 rows (64 a wave), or 128, which take two thirds of the time:
// few rows or heads are done sooner, many cost a third more.  Costs in 0.04 us of
// a streamed tile ([D = 128][own tile][keys]), of a work-group's other work (own
// rows, first loads, stores) and of the merge's launch; a partial of 256 x 128,
// written and read, is 1.  (Splits at 1.5 and a merge at 100: one head of five
// references 365 us, 323 with these.)
constexpr int kBwdOwn[2] = {256, 128};
constexpr int kBwdTile[2][2][2] = {{{34, 36}, {20, 22}}, {{50, 56}, {34, 38}}};
constexpr int kBwdFixed[2][2] = {{80, 60}, {110, 80}};
constexpr int kBwdMerge = 70;

// The schedule of the attention gradient for bh (batch, head)s, from the plans of
// full recomputes of the layout and of its keys.
rc_status plan_bwd(const rc_layout* L, int64_t bh, int32_t D, BwdParams& b) {
  const rc_layout kl = key_layout(L);
  constexpr int kMax = 2 * RC_MAX_SEGMENTS;
  BwdSeg seg[kMax];
  int64_t tiles[kMax];  // streamed tiles of an own tile
  int n = 0;
  for (int keys = 0; keys < 2; ++keys) {
    Params p;
    memset(&p, 0, sizeof p);
    p.bm = kBwdOwn[0];
    RC_TRY(plan(keys ? &kl : L, RC_ENTRY_FULL, p));
    const int first = n;
    for (int i = 0; i < kMaxRanges; ++i)
      b.range[keys * kMaxRanges + i] = BwdRange{p.range[i].start, p.range[i].len};
    for (int i = 0; i < p.n_qseg; ++i) {
      const QSeg& q = p.qseg[i];
      // own segments that follow each other and meet the same rows are one
      BwdSeg* last = n > first ? &seg[n - 1] : nullptr;
      if (last && last->row0 + last->len == q.row0 && last->nr == q.nr &&
          (q.nr == 0 || last->r0 == keys * kMaxRanges + q.r0)) {
        last->len += q.len;
        continue;
      }
      tiles[n] = q.ktiles;
      seg[n++] = BwdSeg{q.row0, q.len, 0, keys * kMaxRanges + q.r0, q.nr, keys, 1, 0};
    }
  }
  // The own tile, and pieces of at most `most` of its streamed tiles, so that few
  // heads fill the chip.  The launch ends with its longest work-group, or with the
  // work spread over the CUs (where first loads and stores half hide) and a part of
  // one.  Drawn sizes of 26 to 5100 rows and 1 to 24 heads: 41 us in the geometric mean with
  // whole 256-row tiles, 34.0 with pieces, 28.9 with 128-row tiles too.
  int64_t longest = 1;
  for (int i = 0; i < n; ++i) longest = std::max(longest, tiles[i]);
  const auto splits_of = [&](int i, int64_t most) { return std::max<int64_t>(1, (tiles[i] + most - 1) / most); };
  const auto cost_of = [&](int i, int64_t most, int own) {
    const int64_t s = splits_of(i, most);
    return (tiles[i] + s - 1) / s * kBwdTile[D == 128][own][seg[i].keys];
  };
  int64_t best = INT64_MAX, best_most = longest;
  int best_own = 0;
  for (int own = 0; own < 2; ++own) {
    for (int64_t s = 1; s <= 32 && (s == 1 || (longest + s - 1) / s >= 2); ++s) {
      const int64_t most = (longest + s - 1) / s;
      int64_t top = 0, total = 0, slots = 0;
      for (int i = 0; i < n; ++i) {
        const int64_t k = splits_of(i, most), c = cost_of(i, most, own);
        const int64_t count = bh * ((seg[i].len + kBwdOwn[own] - 1) / kBwdOwn[own]);
        top = std::max(top, c);
        total += count * k * (c + kBwdFixed[D == 128][own] / 2);
        if (k > 1) slots += count * k * (1 + seg[i].keys);
      }
      top += kBwdFixed[D == 128][own];
      int64_t est = std::max(top, total / kCUs + top / 3);
      if (s > 1) est += kBwdMerge + slots * D * kBwdOwn[own] / (256 * 128);
      const bool plain = best_most == longest && best_own == 0;  // another form has to gain 10%
      if ((s == 1 && own == 0) || est * 10 < best * (plain ? 9 : 10)) best = est, best_most = most, best_own = own;
    }
  }
  b.own = kBwdOwn[best_own];
  // Work-groups run in this order: the longest first, so that the launch ends
  // with short ones (in the order of the segments, queries after keys: 512-pixel
  // edit 348 us, longest first 324).
  int order[kMax];
  for (int i = 0; i < n; ++i) order[i] = i;
  std::sort(order, order + n, [&](int x, int y) {
    const int64_t cx = cost_of(x, best_most, best_own), cy = cost_of(y, best_most, best_own);
    return cx != cy ? cx > cy : x < y;
  });
  b.n_seg = n;
  b.n_pieces = b.n_slots = 0;
  for (int i = 0; i < n; ++i) {
    BwdSeg& g = b.seg[i];
    g = seg[order[i]];
    const int own = (g.len + b.own - 1) / b.own;
    g.splits = int32_t(splits_of(order[i], best_most));
    g.piece0 = b.n_pieces;
    b.n_pieces += own * g.splits;
    g.slot0 = b.n_slots;
    if (g.splits > 1) b.n_slots += own * g.splits * (1 + g.keys);
  }
  return RC_OK;
}

// A launch's threads are counted in 32 bits.
rc_status check_threads(int64_t blocks, int64_t threads, const char* what) {
  if (blocks > ((int64_t(1) << 32) - 1) / threads) {
    set_error("%s launch of %lld x %lld threads exceeds the grid limit", what, (long long)blocks, (long long)threads);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

// lse / scale is a first addend of the recomputed scores and has to stay finite.
constexpr float kBwdMinScale = 0x1p-96f;

// The schedule of a call whose launches stay in their limits.  Rows first: they
// bound the planner's costs, which overflow 64 bits at sizes that B, H and N alone allow.
rc_status plan_bwd_launches(const rc_layout* L, int32_t B, int32_t H, int32_t D, BwdParams& p) {
  const int64_t bh = int64_t(B) * H, rows = bh * count_rows(L, RowSet::All);
  RC_TRY(check_threads((rows * (D / 8) + 255) / 256, 256, "attention gradient"));
  RC_TRY(plan_bwd(L, bh, D, p));
  return check_threads(bh * p.n_pieces, 256, "attention gradient");
}

size_t bwd_partial_bytes(const BwdParams& p, int64_t bh, int32_t D) {
  return size_t(bh) * p.n_slots * p.own * D * sizeof(float);
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

rc_status check_float_ptr(const float* p, const char* name) { return check_lse(p, name); }

bool rotary_size(int32_t B, int64_t N) { return B >= 1 && B <= 65535 && N >= 0 && N <= (int64_t(1) << 31) / B - 1; }

// What both directions of the rotation check, and the parameters they share.
rc_status rotary_params(const rc_rotary* R, int32_t B, int64_t N, int32_t H, const void* a, const void* b,
                        const char* names, const void* positions, int32_t pos_float, int32_t pos_batch,
                        const void* q_norm, const void* k_norm, float eps, RotaryParams& p) {
  if (!R || R->n_axes < 1 || R->n_axes > RC_MAX_ROTARY_AXES || R->width < 0 || R->width > R->head_dim) {
    set_error("rotary: the description is not one that rc_rotary_init has filled");
    return RC_ERR_ARG;
  }
  if (R->head_dim != 64 && R->head_dim != 128) {
    set_error("head_dim %d is not supported (64 or 128)", R->head_dim);
    return RC_ERR_UNSUPPORTED;
  }
  if (!rotary_size(B, N) || H < 1 || H > 65535) {
    set_error("B = %d, H = %d: each must be in [1, 65535]; N = %lld: B * N below 2^31", B, H, (long long)N);
    return RC_ERR_ARG;
  }
  if (N > 0 && !a && !b) {
    set_error("%s are both null", names);
    return RC_ERR_ARG;
  }
  if ((q_norm || k_norm) && !(eps >= 0.f && isfinite(eps))) {
    set_error("eps must be finite and >= 0 (got %g)", (double)eps);
    return RC_ERR_ARG;
  }
  if (N > 0 && ((q_norm && !a) || (k_norm && !b))) {
    set_error("a norm without its tensor");
    return RC_ERR_ARG;
  }
  if (q_norm) RC_TRY(check_ptr(q_norm, "q_norm"));
  if (k_norm) RC_TRY(check_ptr(k_norm, "k_norm"));
  if (N > 0) {
    if (!positions || (reinterpret_cast<uintptr_t>(positions) & 3u)) {
      set_error("positions is null or not 4-byte aligned");
      return RC_ERR_ARG;
    }
  }
  memset(&p, 0, sizeof p);
  p.pos = positions;
  p.pos_float = pos_float != 0;
  p.pos_sb = pos_batch ? N * R->n_axes : 0;
  p.w[0] = static_cast<const uint16_t*>(q_norm);
  p.w[1] = static_cast<const uint16_t*>(k_norm);
  p.N = N;
  p.B = B;
  p.H = H;
  p.axes = R->n_axes;
  p.eps = eps;
  p.width = R->width;
  p.half = R->interleaved ? 0 : R->width / 2;
  for (int i = 0; i < R->head_dim / 2; ++i) {
    const bool in = 2 * i < R->width;
    if (in && (R->axis[i] >= R->n_axes || !isfinite(R->turns[i]))) {
      set_error("rotary: the description is not one that rc_rotary_init has filled");
      return RC_ERR_ARG;
    }
    p.axis[i] = in ? R->axis[i] : 0;
    p.turns[i] = in ? R->turns[i] : 0.0;
  }
  return RC_OK;
}

// Row groups per wave: whole tokens (their sines are computed once) as long as
// that leaves 16 waves per CU, fewer for few tokens.  4608 tokens of 24 heads take
// 20.6 us with 16 waves, 24.7 with 64; 512 tokens 11.4 with either.  At most 12, as
// measured where a token has more: 16384 tokens of 40 heads of 128, 20 groups a token, take
// 124.6 us in waves of 12 and 8, 130.7 in one of 20, 129.3 in waves of 6; 64 heads of 64
// 96.2, 98.7 and 101.6 (4608 tokens of 40 heads 40.8, 40.3 and 39.9); 24 heads of 128, 12
// groups, 76.3 and, in waves of 6, 78.1.
int32_t rotary_groups(const RotaryParams& p, int32_t D) {
  const int rw = 512 / D;
  const int64_t all = int64_t(p.H + rw - 1) / rw * (p.x[0] && p.x[1] ? 2 : 1);
  const int64_t g = all * p.N * p.B / (16 * kCUs);
  return int32_t(std::max<int64_t>(1, std::min<int64_t>({g, all, 12})));
}

int64_t rotary_splits(const RotaryParams& p, int32_t D) {  // waves per token
  const int rw = 512 / D;
  return (int64_t(p.H + rw - 1) / rw * (p.x[0] && p.x[1] ? 2 : 1) + p.groups - 1) / p.groups;
}

int32_t rotary_blocks(int32_t B, int64_t N) {
  return int32_t(std::max<int64_t>(1, std::min<int64_t>(kRotaryBlocks, (N * B + 3) / 4)));
}

rc_status check_rows(const void* ptr, int64_t ld, int32_t C, const char* name) {
  RC_TRY(check_ptr(ptr, name));
  if (ld < C || (ld & 7) || ld > (int64_t(1) << 22)) {
    set_error("%s: row stride %lld must be >= C = %d, a multiple of 8, <= 2^22", name, (long long)ld, C);
    return RC_ERR_ARG;
  }
  return RC_OK;
}

// Checks a gated norm's description and fills what both directions share.
rc_status norm_params(const rc_norm* d, NormParams& p) {
  memset(&p, 0, sizeof p);
  if (!d) {
    set_error("the description is null");
    return RC_ERR_ARG;
  }
  if (d->B < 1 || d->B > 65535 || d->N < 0 || d->N > (int64_t(1) << 31) / d->B - 1 || d->C < 8 || d->C > kNormMaxC ||
      d->C % 8 != 0) {
    set_error("B = %d must be in [1, 65535], B * N below 2^31 (N = %lld), C = %d a multiple of 8 in [8, %d]", d->B,
              (long long)d->N, d->C, kNormMaxC);
    return RC_ERR_ARG;
  }
  if (d->n_groups < 1 || d->n_groups > 65535 || d->n_spans < 0 || d->n_spans > RC_MAX_SEGMENTS ||
      (d->norm != RC_NORM_LAYER && d->norm != RC_NORM_RMS)) {
    set_error("n_groups = %d, n_spans = %d, norm = %d: out of range", d->n_groups, d->n_spans, d->norm);
    return RC_ERR_ARG;
  }
  if (!(d->eps >= 0.f && isfinite(d->eps)) || !isfinite(d->residual_scale)) {
    set_error("eps must be finite and >= 0, residual_scale finite (got %g, %g)", (double)d->eps,
              (double)d->residual_scale);
    return RC_ERR_ARG;
  }
  if (d->mod_batch < 0 || d->mod_group < 0 || (d->mod_batch & 7) || (d->mod_group & 7)) {
    set_error("mod strides %lld, %lld must be multiples of 8, >= 0", (long long)d->mod_batch, (long long)d->mod_group);
    return RC_ERR_ARG;
  }
  int64_t n = 0;
  for (int s = 0; s < d->n_spans; ++s) {
    if (d->rows[s] < 0 || d->group[s] < 0 || d->group[s] >= d->n_groups) {
      set_error("span %d: %d rows of group %d (of %d)", s, d->rows[s], d->group[s], d->n_groups);
      return RC_ERR_ARG;
    }
    if (d->rows[s] == 0) continue;
    p.span_row0[p.n_spans] = int32_t(std::min<int64_t>(n, INT32_MAX));
    p.span_rows[p.n_spans] = d->rows[s];
    p.span_group[p.n_spans++] = d->group[s];
    n += d->rows[s];
  }
  if (n != d->N) {
    set_error("the spans have %lld rows, the batch entries %lld", (long long)n, (long long)d->N);
    return RC_ERR_ARG;
  }
  p.mod_sb = d->mod_batch;
  p.mod_sg = d->mod_group;
  p.N = d->N;
  p.B = d->B;
  p.C = d->C;
  p.G = d->n_groups;
  p.rms = d->norm == RC_NORM_RMS;
  p.post = d->post != 0;
  p.eps = d->eps;
  p.rscale = d->residual_scale;
  p.inv_c = 1.f / float(d->C);
  // The backward's chunks, one work-group each and one work-group per CU:
  // rows per chunk such that all of them fit one round (every span ends with a
  // shorter one).  A multiple of four: a work-group takes four rows together where a row
  // has 129 to 384 granules of 8 channels, eight below (the last step of a chunk may then be
  // half empty), two or one above.
  const int64_t rows = d->N * d->B;
  // Where entries and spans alone are more, a span is one chunk.
  int64_t per = std::max<int64_t>(8, (rows + kCUs - 1) / kCUs + 3) / 4 * 4;
  for (;; per += std::max<int64_t>(4, per / 64 / 4 * 4)) {
    int64_t n_chunks = 0, longest = 0;
    for (int s = 0; s < p.n_spans; ++s) {
      n_chunks += (p.span_rows[s] + per - 1) / per;
      longest = std::max<int64_t>(longest, p.span_rows[s]);
    }
    if (n_chunks * d->B <= kCUs || per >= longest) break;
  }
  p.chunk_rows = int32_t(std::min<int64_t>(per, INT32_MAX));
  for (int s = 0; s < p.n_spans; ++s) {
    p.span_chunk0[s] = p.chunks;
    p.chunks += (p.span_rows[s] + p.chunk_rows - 1) / p.chunk_rows;
  }
  return RC_OK;
}

rc_status check_vec(const void* p, const char* name) { return p ? check_ptr(p, name) : RC_OK; }

NormRows rows_of(const void* p, int64_t ld) { return NormRows{static_cast<uint16_t*>(const_cast<void*>(p)), ld}; }

size_t norm_partial_bytes(const NormParams& p) { return size_t(p.B) * p.chunks * 3 * p.C * sizeof(float); }

// Per-row statistics of the gradient: two floats per (batch, head, row), each
// in a 16-byte aligned array.
size_t bwd_row_bytes(int64_t rows) { return (size_t(rows) * sizeof(float) + 15) & ~size_t(15); }

}  // namespace
}  // namespace rc

using namespace rc;

extern "C" {

rc_status rc_ref_kv_prefill(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale,
                            const void* q_static, const void* k_static, const void* v_static,
                            int64_t tok_stride, void* o_static, float* lse_static, void* k_cache,
                            void* v_cache, void* stream) {
  return prefill_impl(L, B, H, D, scale, q_static, k_static, v_static, tok_stride, o_static, lse_static, false,
                      k_cache, v_cache, nullptr, stream);
}

rc_status rc_ref_kv_prefill_fp8(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale,
                                const void* q_static, const void* k_static, const void* v_static,
                                int64_t tok_stride, void* o_static, float* lse_static, void* k_cache8,
                                void* v_cache8, float* kv_scale, void* stream) {
  return prefill_impl(L, B, H, D, scale, q_static, k_static, v_static, tok_stride, o_static, lse_static, true,
                      k_cache8, v_cache8, kv_scale, stream);
}

int32_t rc_step_auto_splits(const rc_layout* L, int32_t B, int32_t H, int32_t D) {
  if (check_layout(L, RC_ENTRY_STEP) != RC_OK) return 1;
  if (B < 1 || H < 1 || (D != 64 && D != 128)) return 1;
  Params p;
  memset(&p, 0, sizeof p);
  p.B = B;
  p.H = H;
  p.bm = rows_per_wg(kQBPlain);
  if (plan(L, RC_ENTRY_STEP, p) != RC_OK) return 1;
  return auto_splits(p);
}

rc_status rc_prefill_launch_plan(const rc_layout* L, int32_t B, int32_t H, int32_t D, int64_t* attn_wgs,
                                 int32_t* copy_wgs, int64_t* copy_rows) {
  using namespace rc;
  RC_TRY(check_layout(L, RC_ENTRY_PREFILL));
  if (!attn_wgs || !copy_wgs || !copy_rows) {
    set_error("rc_prefill_launch_plan: null output pointer");
    return RC_ERR_ARG;
  }
  RC_TRY(check_dims(B, H, D, 1.0f));
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, 1.0f);
  RC_TRY(plan_prefill(L, D, false, p));
  *attn_wgs = int64_t(B) * H * p.n_qtiles;
  *copy_wgs = p.cp.blocks;
  *copy_rows = p.cp.rows;
  return RC_OK;
}

rc_status rc_step_launch_shape(const rc_layout* L, int32_t B, int32_t H, int32_t D, int32_t splits, int32_t fp8,
                               int64_t* work_groups, int32_t* rows_per_wg, int32_t* splits_used) {
  using namespace rc;
  RC_TRY(check_layout(L, RC_ENTRY_STEP));
  if (!work_groups || !rows_per_wg || !splits_used) {
    set_error("rc_step_launch_shape: null output pointer");
    return RC_ERR_ARG;
  }
  RC_TRY(check_dims(B, H, D, 1.0f));
  if (splits < kSplitsLastRound || splits > kMaxSplits || (fp8 != 0 && fp8 != 1)) {
    set_error("rc_step_launch_shape: splits = %d or fp8 = %d out of range", splits, fp8);
    return RC_ERR_ARG;
  }
  if (fp8 && splits == kSplitsBalanced) {
    set_error("the balanced schedule is not available with the FP8 cache");
    return RC_ERR_UNSUPPORTED;
  }
  Params p;
  memset(&p, 0, sizeof p);
  p.B = B;
  p.H = H;
  RC_TRY(plan_step(L, D, fp8 != 0, splits, p));
  *rows_per_wg = p.bm;
  *splits_used = p.splits;
  if (p.lr_tiles > 0) *splits_used = kSplitsLastRound;
  *work_groups = p.splits == kSplitsBalanced ? int64_t(p.bal_wgs)
                 : p.lr_tiles > 0            ? int64_t(B) * H * p.n_qtiles + p.lr_tiles
                                             : int64_t(B) * H * p.n_qtiles * p.splits;
  return RC_OK;
}

int64_t rc_attention_work_groups(const rc_layout* L, int32_t entry, int32_t B, int32_t H, int32_t D, int32_t splits,
                                 int32_t fp8) {
  using namespace rc;
  RC_TRY(check_layout(L, entry));
  RC_TRY(check_dims(B, H, D, 1.0f));
  if (fp8 != 0 && fp8 != 1) {
    set_error("rc_attention_work_groups: fp8 = %d must be 0 or 1", fp8);
    return RC_ERR_ARG;
  }
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, 1.0f);
  if (entry == RC_ENTRY_STEP) {
    int64_t wgs;
    int32_t bm, used;
    RC_TRY(rc_step_launch_shape(L, B, H, D, splits, fp8, &wgs, &bm, &used));  // checks splits
    RC_TRY(plan_step(L, D, fp8 != 0, splits, p));
  } else if (splits != 1 && !(entry == RC_ENTRY_FULL && splits == kSplitsLastRound)) {
    set_error("rc_attention_work_groups: splits = %d", splits);
    return RC_ERR_ARG;
  } else if (entry == RC_ENTRY_FULL) {
    RC_TRY(plan_full(L, splits == kSplitsLastRound, p));
  } else {
    RC_TRY(plan_prefill(L, D, fp8 != 0, p));
  }
  return attention_work_groups(p);
}

size_t rc_step_workspace_bytes(const rc_layout* L, int32_t B, int32_t H, int32_t D, int32_t splits) {
  if (check_layout(L, RC_ENTRY_STEP) != RC_OK) return 0;
  if (B < 1 || H < 1 || (D != 64 && D != 128) || splits < kSplitsLastRound || splits > kMaxSplits) return 0;
  if (splits == 0) splits = rc_step_auto_splits(L, B, H, D);
  if (splits == kSplitsBalanced) return balanced_workspace_bytes(D);
  if (splits == kSplitsLastRound) {
    Params p;
    memset(&p, 0, sizeof p);
    p.B = B;
    p.H = H;
    p.bm = rows_per_wg(kQBPlain);
    if (plan(L, RC_ENTRY_STEP, p) != RC_OK) return 0;
    return size_t(2) * last_round_tiles(p) * p.bm * size_t(D + 2) * sizeof(float);
  }
  if (splits == kSplitsTail) splits = 2;
  if (splits <= 1) return 0;
  const int64_t n_live = count_rows(L, RowSet::Live);
  return size_t(splits) * size_t(B) * size_t(H) * size_t(n_live) * size_t(D + 2) * sizeof(float);
}

rc_status rc_step_masked_attention(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale,
                                   const void* q_live, const void* k_live, const void* v_live,
                                   int64_t tok_stride, const void* k_cache, const void* v_cache,
                                   void* o_live, float* lse_live, int32_t splits, void* workspace,
                                   size_t ws_bytes, void* stream) {
  return step_impl(L, B, H, D, scale, q_live, k_live, v_live, tok_stride, false, k_cache, v_cache, nullptr, o_live,
                   lse_live, splits, workspace, ws_bytes, stream);
}

rc_status rc_step_masked_attention_noalloc(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale,
                                           const void* q_live, const void* k_live, const void* v_live,
                                           int64_t tok_stride, const void* k_cache, const void* v_cache,
                                           void* o_live, float* lse_live, int32_t splits, void* stream) {
  using namespace rc;
  // the workspace the split choice needs (0 for none, or for invalid input,
  // which step_impl then reports)
  const size_t need = rc_step_workspace_bytes(L, B, H, D, splits);
  if (need > size_t(RC_NOALLOC_SCRATCH_BYTES)) {
    set_error("the no-allocation step holds %zu bytes of scratch; splits = %d needs %zu",
              size_t(RC_NOALLOC_SCRATCH_BYTES), splits, need);
    return RC_ERR_WORKSPACE;
  }
  void* ws = nullptr;
  if (need > 0) RC_TRY(hip_status(scratch_address(&ws), "scratch lookup"));
  return step_impl(L, B, H, D, scale, q_live, k_live, v_live, tok_stride, false, k_cache, v_cache, nullptr, o_live,
                   lse_live, splits, ws, need > 0 ? size_t(RC_NOALLOC_SCRATCH_BYTES) : 0, stream);
}

rc_status rc_step_masked_attention_fp8(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale,
                                       const void* q_live, const void* k_live, const void* v_live,
                                       int64_t tok_stride, const void* k_cache8, const void* v_cache8,
                                       const float* kv_scale, void* o_live, float* lse_live, int32_t splits,
                                       void* workspace, size_t ws_bytes, void* stream) {
  return step_impl(L, B, H, D, scale, q_live, k_live, v_live, tok_stride, true, k_cache8, v_cache8, kv_scale,
                   o_live, lse_live, splits, workspace, ws_bytes, stream);
}

size_t rc_full_workspace_bytes(const rc_layout* L, int32_t B, int32_t H, int32_t D) {
  using namespace rc;
  if (B < 1 || H < 1 || (D != 64 && D != 128)) return 0;
  if (check_layout(L, RC_ENTRY_FULL) != RC_OK) return 0;
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, 1.0f);
  p.bm = rows_per_wg(kQBPlain);
  if (plan(L, RC_ENTRY_FULL, p) != RC_OK) return 0;
  return size_t(2) * last_round_tiles(p) * p.bm * size_t(D + 2) * sizeof(float);
}

rc_status rc_full_attention_ws(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale, const void* q,
                               const void* k, const void* v, int64_t tok_stride, void* o, float* lse,
                               void* workspace, size_t ws_bytes, void* stream) {
  RC_TRY(check_layout(L, RC_ENTRY_FULL));
  RC_TRY(check_dims(B, H, D, scale));
  RC_TRY(check_stride(tok_stride, H, D));
  RC_TRY(check_ptr(q, "q"));
  RC_TRY(check_ptr(k, "k"));
  RC_TRY(check_ptr(v, "v"));
  RC_TRY(check_ptr(o, "o"));
  RC_TRY(check_lse(lse, "lse"));
  const int64_t n = count_rows(L, RowSet::All);
  Params p;
  memset(&p, 0, sizeof p);
  fill_common(p, B, H, scale);
  RC_TRY(plan_full(L, workspace != nullptr, p));
  // the grid unsplit: the last-round split adds its pieces below
  RC_TRY(check_blocks(int64_t(B) * H * p.n_qtiles, "attention"));
  p.q = static_cast<const uint16_t*>(q);
  p.q_st = tok_stride;
  p.q_sb = tok_stride * n;
  p.o = static_cast<uint16_t*>(o);
  p.o_st = int64_t(H) * D;
  p.o_sb = p.o_st * n;
  p.lse = lse;
  p.src[0] = bf16_source(k, v, tok_stride * n, D, tok_stride);
  const int32_t T = p.lr_tiles;
  if (workspace) {
    const size_t need = size_t(2) * T * p.bm * size_t(D + 2) * sizeof(float);
    if (!aligned16(workspace) || ws_bytes < need) {
      set_error("the last-round split needs a 16-byte aligned workspace of %zu bytes (got %zu)", need, ws_bytes);
      return RC_ERR_WORKSPACE;
    }
  }
  if (T > 0) {
    p.ws_o = static_cast<float*>(workspace);
    p.ws_ml = p.ws_o + size_t(2) * T * p.bm * D;
    RC_TRY(check_blocks(int64_t(B) * H * p.n_qtiles + T, "full attention"));
  }
  RC_TRY(hip_status(launch_attention(p, D, stream), "full attention launch"));
  if (T > 0) RC_TRY(hip_status(launch_combine_last_round(p, D, stream), "last-round merge launch"));
  return RC_OK;
}

rc_status rc_full_attention(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale, const void* q,
                            const void* k, const void* v, int64_t tok_stride, void* o, float* lse,
                            void* stream) {
  return rc_full_attention_ws(L, B, H, D, scale, q, k, v, tok_stride, o, lse, nullptr, 0, stream);
}

rc_status rc_linear(int64_t M, int32_t N, int32_t K, const void* a, int64_t lda, const void* w, const void* r,
                    int64_t ldr, void* out, int64_t ldo, void* stream) {
  if (M < 0 || M > (int64_t(1) << 40) || N <= 0 || K <= 0) {
    set_error("linear: M = %lld, N = %d, K = %d must be in [0, 2^40], > 0, > 0", (long long)M, N, K);
    return RC_ERR_ARG;
  }
  if (N % 128 != 0 || K % 64 != 0 || K > (1 << 22)) {
    set_error("linear: N = %d must be a multiple of 128 and K = %d a multiple of 64 up to 2^22", N, K);
    return RC_ERR_UNSUPPORTED;
  }
  const auto bad_ld = [](int64_t ld, int64_t lo) { return ld < lo || ld % 8 != 0 || ld > (int64_t(1) << 22); };
  if (bad_ld(lda, K) || bad_ld(ldo, N) || (r && bad_ld(ldr, N))) {
    set_error("linear: strides lda = %lld, ldr = %lld, ldo = %lld must be >= K / N, multiples of 8, <= 2^22",
              (long long)lda, (long long)ldr, (long long)ldo);
    return RC_ERR_ARG;
  }
  if (M == 0) return RC_OK;
  RC_TRY(check_ptr(a, "a"));
  RC_TRY(check_ptr(w, "w"));
  RC_TRY(check_ptr(out, "out"));
  if (r) RC_TRY(check_ptr(r, "r"));
  RC_TRY(check_blocks((M + 127) / 128 * (N / 128), "linear"));
  LinearParams q;
  q.a = static_cast<const uint16_t*>(a);
  q.w = static_cast<const uint16_t*>(w);
  q.r = static_cast<const uint16_t*>(r);
  q.out = static_cast<uint16_t*>(out);
  q.M = M;
  q.N = N;
  q.K = K;
  q.lda = lda;
  q.ldr = r ? ldr : 0;
  q.ldo = ldo;
  RC_TRY(hip_status(launch_linear(q, stream), "linear launch"));
  return RC_OK;
}

size_t rc_full_backward_workspace_bytes(const rc_layout* L, int32_t B, int32_t H, int32_t D) {
  if (B < 1 || H < 1 || B > 65535 || H > 65535 || (D != 64 && D != 128)) return 0;
  if (check_layout(L, RC_ENTRY_FULL) != RC_OK) return 0;
  BwdParams p;
  const int64_t bh = int64_t(B) * H;
  if (plan_bwd_launches(L, B, H, D, p) != RC_OK) return 0;
  return 2 * bwd_row_bytes(bh * count_rows(L, RowSet::All)) + bwd_partial_bytes(p, bh, D);
}

rc_status rc_full_attention_backward(const rc_layout* L, int32_t B, int32_t H, int32_t D, float scale, const void* q,
                                     const void* k, const void* v, int64_t tok_stride, const void* o,
                                     const float* lse, const void* d_o, const float* dlse, void* dq, void* dk,
                                     void* dv, int64_t grad_stride, void* workspace, size_t ws_bytes, void* stream) {
  RC_TRY(check_layout(L, RC_ENTRY_FULL));
  RC_TRY(check_dims(B, H, D, scale));
  if (scale < kBwdMinScale) {
    set_error("softmax scale %g: the attention gradient takes 2^-96 and more", (double)scale);
    return RC_ERR_UNSUPPORTED;
  }
  RC_TRY(check_stride(tok_stride, H, D));
  RC_TRY(check_stride(grad_stride, H, D));
  RC_TRY(check_stride(int64_t(H) * D, H, D));  // O and dO
  RC_TRY(check_ptr(q, "q"));
  RC_TRY(check_ptr(k, "k"));
  RC_TRY(check_ptr(v, "v"));
  RC_TRY(check_ptr(o, "o"));
  RC_TRY(check_ptr(d_o, "d_o"));
  if (!lse) {
    set_error("lse is null");
    return RC_ERR_ARG;
  }
  RC_TRY(check_lse(lse, "lse"));
  RC_TRY(check_lse(dlse, "dlse"));
  RC_TRY(check_ptr(dq, "dq"));
  RC_TRY(check_ptr(dk, "dk"));
  RC_TRY(check_ptr(dv, "dv"));
  const int64_t n = count_rows(L, RowSet::All), rows = int64_t(B) * H * n;
  BwdParams p;
  memset(&p, 0, sizeof p);
  RC_TRY(plan_bwd_launches(L, B, H, D, p));
  const size_t need = 2 * bwd_row_bytes(rows) + bwd_partial_bytes(p, int64_t(B) * H, D);
  if (!workspace || !aligned16(workspace) || ws_bytes < need) {
    set_error("the attention gradient needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
              workspace ? ws_bytes : size_t(0));
    return RC_ERR_WORKSPACE;
  }
  RC_TRY(check_launcher(launch_attention_bwd, "attention gradient"));
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<const uint16_t*>(o);
  p.d_o = static_cast<const uint16_t*>(d_o);
  p.lse = lse;
  p.dlse = dlse;
  p.dq = static_cast<uint16_t*>(dq);
  p.dk = static_cast<uint16_t*>(dk);
  p.dv = static_cast<uint16_t*>(dv);
  p.nlse = static_cast<float*>(workspace);
  p.ndelta = p.nlse + bwd_row_bytes(rows) / sizeof(float);
  p.partial = p.ndelta + bwd_row_bytes(rows) / sizeof(float);
  p.st = tok_stride;
  p.g_st = grad_stride;
  p.B = B;
  p.H = H;
  p.n_rows = int32_t(n);
  p.scale = scale;
  p.scale_log2 = scale * 1.4426950408889634f;
  RC_TRY(hip_status(launch_attention_bwd(p, D, stream), "attention gradient launch"));
  return RC_OK;
}

rc_status rc_rotary_init(rc_rotary* R, int32_t head_dim, int32_t n_axes, const int32_t* axes, double theta,
                         int32_t interleaved, int32_t continuous) {
  if (!R || !axes || n_axes < 1 || n_axes > RC_MAX_ROTARY_AXES) {
    set_error("rotary: null argument, or n_axes = %d not in [1, %d]", n_axes, RC_MAX_ROTARY_AXES);
    return RC_ERR_ARG;
  }
  if (head_dim != 64 && head_dim != 128) {
    set_error("head_dim %d is not supported (64 or 128)", head_dim);
    return RC_ERR_UNSUPPORTED;
  }
  if (!(theta > 0.0) || !isfinite(theta)) {
    set_error("theta must be finite and > 0 (got %g)", theta);
    return RC_ERR_ARG;
  }
  int64_t width = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (axes[a] < 0 || axes[a] % 2 != 0 || (width += axes[a]) > head_dim) {
      set_error("axis %d: width %d must be even, and the widths add up to at most %d", a, axes[a], head_dim);
      return RC_ERR_ARG;
    }
  }
  if (!interleaved && width % 16 != 0) {
    set_error("pairs of halves need a rotated width that is a multiple of 16 (got %lld)", (long long)width);
    return RC_ERR_UNSUPPORTED;
  }
  memset(R, 0, sizeof *R);
  R->head_dim = head_dim;
  R->n_axes = n_axes;
  R->width = int32_t(width);
  R->interleaved = interleaved != 0;
  int p = 0;
  for (int a = 0; a < n_axes; ++a)
    for (int i = 0; i < axes[a] / 2; ++i, ++p) {
      const double e = continuous ? 2.0 * p / double(width) : 2.0 * i / double(axes[a]);
      R->axis[p] = uint8_t(a);
      R->turns[p] = pow(theta, -e) / kTwoPi;
    }
  return RC_OK;
}

rc_status rc_qk_rotary(const rc_rotary* R, int32_t B, int64_t N, int32_t H, const void* q, const void* k,
                       int64_t tok_stride, const void* positions, int32_t pos_float, int32_t pos_batch,
                       const void* q_norm, const void* k_norm, float eps, void* q_out, void* k_out,
                       int64_t out_stride, void* stream) {
  RotaryParams p;
  RC_TRY(rotary_params(R, B, N, H, q, k, "q and k", positions, pos_float, pos_batch, q_norm, k_norm, eps, p));
  const int32_t D = R->head_dim;
  RC_TRY(check_stride(tok_stride, H, D));
  RC_TRY(check_stride(out_stride, H, D));
  if (N == 0) return RC_OK;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    RC_TRY(check_ptr(in[i], i ? "k" : "q"));
    RC_TRY(check_ptr(out[i], i ? "k_out" : "q_out"));
    if (in[i] == out[i] && tok_stride != out_stride) {
      set_error("%s in place needs the input's token stride", i ? "k" : "q");
      return RC_ERR_ARG;
    }
    p.x[i] = static_cast<const uint16_t*>(in[i]);
    p.y[i] = static_cast<uint16_t*>(out[i]);
  }
  p.x_st = tok_stride;
  p.y_st = out_stride;
  p.sign = 1.f;
  p.groups = rotary_groups(p, D);
  RC_TRY(check_threads((B * N * rotary_splits(p, D) + 3) / 4, 256, "rotation"));
  RC_TRY(check_launcher(launch_rotary, "rotation"));
  RC_TRY(hip_status(launch_rotary(p, D, stream), "rotation launch"));
  return RC_OK;
}

size_t rc_rotary_backward_workspace_bytes(const rc_rotary* R, int32_t B, int64_t N) {
  if (!R || (R->head_dim != 64 && R->head_dim != 128) || !rotary_size(B, N)) return 0;
  return size_t(rotary_blocks(B, N)) * 2 * R->head_dim * sizeof(float);
}

rc_status rc_qk_rotary_backward(const rc_rotary* R, int32_t B, int64_t N, int32_t H, const void* dq, const void* dk,
                                int64_t grad_stride, const void* positions, int32_t pos_float, int32_t pos_batch,
                                const void* q, const void* k, int64_t tok_stride, const void* q_norm,
                                const void* k_norm, float eps, void* dq_in, void* dk_in, int64_t out_stride,
                                float* dq_norm, float* dk_norm, void* workspace, size_t ws_bytes, void* stream) {
  RotaryParams p;
  RC_TRY(rotary_params(R, B, N, H, dq, dk, "dq and dk", positions, pos_float, pos_batch, q_norm, k_norm, eps, p));
  const int32_t D = R->head_dim;
  const bool norm = q_norm || k_norm;
  RC_TRY(check_stride(grad_stride, H, D));
  RC_TRY(check_stride(out_stride, H, D));
  if (norm) RC_TRY(check_stride(tok_stride, H, D));
  if ((dq_norm && !q_norm) || (dk_norm && !k_norm)) {
    set_error("the gradient of a norm that is not there");
    return RC_ERR_ARG;
  }
  RC_TRY(check_float_ptr(dq_norm, "dq_norm"));
  RC_TRY(check_float_ptr(dk_norm, "dk_norm"));
  const void* g[2] = {dq, dk};
  const void* n[2] = {q, k};
  void* out[2] = {dq_in, dk_in};
  for (int i = 0; i < 2 && N > 0; ++i) {
    if (!g[i]) continue;
    RC_TRY(check_ptr(g[i], i ? "dk" : "dq"));
    RC_TRY(check_ptr(out[i], i ? "dk_in" : "dq_in"));
    if (p.w[i]) RC_TRY(check_ptr(n[i], i ? "k" : "q"));
    if (g[i] == out[i] && grad_stride != out_stride) {
      set_error("%s in place needs the input's token stride", i ? "dk" : "dq");
      return RC_ERR_ARG;
    }
    p.x[i] = static_cast<const uint16_t*>(g[i]);
    p.n[i] = static_cast<const uint16_t*>(n[i]);
    p.y[i] = static_cast<uint16_t*>(out[i]);
  }
  p.x_st = grad_stride;
  p.n_st = tok_stride;
  p.y_st = out_stride;
  p.sign = -1.f;
  if (!norm) {
    if (N == 0) return RC_OK;
    p.groups = rotary_groups(p, D);
    RC_TRY(check_threads((B * N * rotary_splits(p, D) + 3) / 4, 256, "rotation gradient"));
    RC_TRY(check_launcher(launch_rotary, "rotation gradient"));
    RC_TRY(hip_status(launch_rotary(p, D, stream), "rotation gradient launch"));
    return RC_OK;
  }
  const size_t need = rc_rotary_backward_workspace_bytes(R, B, N);
  if (!workspace || !aligned16(workspace) || ws_bytes < need) {
    set_error("the rotation's gradient with a norm needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
              workspace ? ws_bytes : size_t(0));
    return RC_ERR_WORKSPACE;
  }
  p.partial = static_cast<float*>(workspace);
  p.dw[0] = dq_norm;
  p.dw[1] = dk_norm;
  p.blocks = rotary_blocks(B, N);
  RC_TRY(check_launcher(launch_rotary_norm_backward, "rotation gradient"));
  RC_TRY(hip_status(launch_rotary_norm_backward(p, D, stream), "rotation gradient launch"));
  return RC_OK;
}

rc_status rc_gated_norm(const rc_norm* d, const void* h, int64_t ldh, const void* x, int64_t ldx, const void* gate,
                        const void* scale, const void* shift, const void* weight, const void* post_weight,
                        void* h_out, int64_t ldho, void* y, int64_t ldy, void* stream) {
  NormParams p;
  RC_TRY(norm_params(d, p));
  if (p.N > 0 &&
      ((x == nullptr) != (h_out == nullptr) || (!x && (gate || post_weight || p.post)) || (!x && !y))) {
    set_error("gated norm: x and h_out go together, gate and the norm after the block with x; y without x");
    return RC_ERR_ARG;
  }
  if (post_weight && !p.post) {
    set_error("post_weight without the norm after the block");
    return RC_ERR_ARG;
  }
  if (p.N > 0 && !y && (scale || shift || weight)) {
    set_error("scale, shift and weight belong to y");
    return RC_ERR_ARG;
  }
  if (p.N == 0) return RC_OK;
  RC_TRY(check_rows(h, ldh, p.C, "h"));
  if (x) {
    RC_TRY(check_rows(x, ldx, p.C, "x"));
    RC_TRY(check_rows(h_out, ldho, p.C, "h_out"));
    if (h_out == h && ldho != ldh) {
      set_error("h_out in place needs h's row stride");
      return RC_ERR_ARG;
    }
  }
  if (y) RC_TRY(check_rows(y, ldy, p.C, "y"));
  RC_TRY(check_vec(gate, "gate"));
  RC_TRY(check_vec(scale, "scale"));
  RC_TRY(check_vec(shift, "shift"));
  RC_TRY(check_vec(weight, "weight"));
  RC_TRY(check_vec(post_weight, "post_weight"));
  p.h = rows_of(h, ldh);
  p.x = rows_of(x, ldx);
  p.h_out = rows_of(h_out, ldho);
  p.y = rows_of(y, ldy);
  p.gate = static_cast<const uint16_t*>(gate);
  p.scale = static_cast<const uint16_t*>(scale);
  p.shift = static_cast<const uint16_t*>(shift);
  p.weight = static_cast<const uint16_t*>(weight);
  p.post_weight = static_cast<const uint16_t*>(post_weight);
  RC_TRY(check_threads(p.N * p.B, p.C <= 1024 ? 64 : 256, "gated norm"));
  RC_TRY(check_launcher(launch_norm, "gated norm"));
  RC_TRY(hip_status(launch_norm(p, stream), "gated norm launch"));
  return RC_OK;
}

size_t rc_gated_norm_backward_workspace_bytes(const rc_norm* d) {
  NormParams p;
  return norm_params(d, p) == RC_OK ? norm_partial_bytes(p) : 0;
}

rc_status rc_gated_norm_backward(const rc_norm* d, const void* dy, int64_t lddy, const void* dh, int64_t lddh,
                                 const void* h, int64_t ldh, const void* x, int64_t ldx, const void* gate,
                                 const void* scale, const void* weight, const void* post_weight, void* dh_in,
                                 int64_t lddhi, void* dx, int64_t lddx, float* dgate, float* dscale, float* dshift,
                                 float* dweight, float* dpost_weight, void* workspace, size_t ws_bytes,
                                 void* stream) {
  NormParams p;
  RC_TRY(norm_params(d, p));
  if (p.N > 0 &&
      ((x == nullptr) != (dx == nullptr) || (!x && (gate || post_weight || p.post || dgate || dpost_weight)))) {
    set_error("gated norm: x and dx go together, gate and the norm after the block with x");
    return RC_ERR_ARG;
  }
  if (post_weight && !p.post) {
    set_error("post_weight without the norm after the block");
    return RC_ERR_ARG;
  }
  if (p.N > 0 && ((!dy && (scale || weight || dscale || dshift || dweight)) || (!dy && !dh))) {
    set_error("without dy there is only dh, no scale, shift or weight");
    return RC_ERR_ARG;
  }
  if ((dweight && !weight) || (dpost_weight && !post_weight) || (dgate && !gate)) {
    set_error("the gradient of a vector that is not there");
    return RC_ERR_ARG;
  }
  if (p.N > 0) {
    if (dy) {
      RC_TRY(check_rows(dy, lddy, p.C, "dy"));
      RC_TRY(check_rows(h, ldh, p.C, "h"));
    }
    if (dh) RC_TRY(check_rows(dh, lddh, p.C, "dh"));
    RC_TRY(check_rows(dh_in, lddhi, p.C, "dh_in"));
    if (x) {
      RC_TRY(check_rows(x, ldx, p.C, "x"));
      RC_TRY(check_rows(dx, lddx, p.C, "dx"));
    }
    if ((dh_in == dh && lddhi != lddh) || (dh_in == dy && lddhi != lddy) || (x && dx == x && lddx != ldx)) {
      set_error("a gradient in place needs its input's row stride");
      return RC_ERR_ARG;
    }
  }
  RC_TRY(check_vec(gate, "gate"));
  RC_TRY(check_vec(scale, "scale"));
  RC_TRY(check_vec(weight, "weight"));
  RC_TRY(check_vec(post_weight, "post_weight"));
  if (int64_t(p.B) * p.G >= 65535) {  // a work-group per vector of 64 columns, in the grid's second axis
    set_error("gated norm: the gradients of B * n_groups = %lld vectors (at most 65534)", (long long)p.B * p.G);
    return RC_ERR_UNSUPPORTED;
  }
  const struct {
    const float* p;
    const char* name;
  } outs[] = {{dgate, "dgate"}, {dscale, "dscale"}, {dshift, "dshift"}, {dweight, "dweight"},
              {dpost_weight, "dpost_weight"}};
  for (const auto& o : outs) RC_TRY(check_float_ptr(o.p, o.name));
  const size_t need = norm_partial_bytes(p);
  if (need > 0 && (!workspace || !aligned16(workspace) || ws_bytes < need)) {
    set_error("the gated norm's gradient needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
              workspace ? ws_bytes : size_t(0));
    return RC_ERR_WORKSPACE;
  }
  p.dy = rows_of(dy, lddy);
  p.dh = rows_of(dh, lddh);
  p.h = rows_of(h, ldh);
  p.x = rows_of(x, ldx);
  p.dh_in = rows_of(dh_in, lddhi);
  p.dx = rows_of(dx, lddx);
  p.gate = static_cast<const uint16_t*>(gate);
  p.scale = static_cast<const uint16_t*>(scale);
  p.weight = static_cast<const uint16_t*>(weight);
  p.post_weight = static_cast<const uint16_t*>(post_weight);
  p.dgate = dgate;
  p.dscale = dscale;
  p.dshift = dshift;
  p.dweight = dweight;
  p.dpost_weight = dpost_weight;
  p.partial = static_cast<float*>(workspace);
  RC_TRY(check_launcher(launch_norm_backward, "gated norm gradient"));
  RC_TRY(hip_status(launch_norm_backward(p, stream), "gated norm gradient launch"));
  return RC_OK;
}

}  // extern "C"
