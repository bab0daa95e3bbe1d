"""ctypes binding of librefcache (include/refcache.h).

Argument marshalling only: tensors are passed as device pointers and the
current torch stream as a hipStream_t; every step of the computation runs in
the library's HIP kernels.  torch supplies device memory and streams.

``stream=`` runs a call on that stream instead: as everywhere in torch, the
caller orders it after the work that made the inputs and before the reads of
the outputs, and keeps the tensors it passes until the call's kernels are
done.  What the call allocates itself lives as long as they need it.

Loading fails loudly if the library has not been built
(``python -m paper_2608_21229_amd.build``): there is no fallback path.
"""
from __future__ import annotations

import collections
import ctypes
import math
import os
from typing import Iterable, Optional, Sequence, Tuple

RC_MAX_SEGMENTS = 32
SPLITS_BALANCED = -1   # rc_step_masked_attention: one round of 256 work-groups sharing all key tiles evenly
NOALLOC_SCRATCH_BYTES = 128 << 20   # rc_step_masked_attention_noalloc's static scratch per GPU
SPLITS_TAIL = -2       # rc_step_masked_attention: a long and a short key split per query tile (idle CUs take the short)
SPLITS_LAST_ROUND = -3  # rc_step_masked_attention: the tail split for the query tiles of a grid's partial last round
RC_OK, RC_ERR_ARG, RC_ERR_UNSUPPORTED, RC_ERR_MASK_NOT_CACHEABLE, RC_ERR_WORKSPACE, RC_ERR_HIP = 0, -1, -2, -3, -4, -5
SEG_ANCHOR, SEG_TEXT, SEG_TARGET, SEG_REF = 0, 1, 2, 3
MASK_PAPER, MASK_PERREF, MASK_ISOLATED, MASK_DENSE = 0, 1, 2, 3
ENTRY_PREFILL, ENTRY_STEP, ENTRY_FULL = 0, 1, 2
ROWS_STATIC, ROWS_LIVE, ROWS_CACHED, ROWS_ALL = 0, 1, 2, 3
MASKS = {"paper": MASK_PAPER, "perref": MASK_PERREF, "isolated": MASK_ISOLATED, "dense": MASK_DENSE}

# REFCACHE_LIB names another build of the same ABI (the host tests load a
# sanitizer build of the planner through it); by default the in-tree library.
LIB_PATH = os.environ.get("REFCACHE_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                          "librefcache.so")


class RcError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"librefcache status {status}: {message}")
        self.status = status


class _Segment(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("len", ctypes.c_int32)]


class rc_layout(ctypes.Structure):
    _fields_ = [("n_seg", ctypes.c_int32),
                ("seg", _Segment * RC_MAX_SEGMENTS),
                ("visible", ctypes.c_uint32 * RC_MAX_SEGMENTS)]


class rc_rotary(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("width", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("axis", ctypes.c_uint8 * 64), ("turns", ctypes.c_double * 64)]


class rc_blocks8(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("ld", ctypes.c_int64), ("exps", ctypes.c_void_p),
                ("ld_exps", ctypes.c_int64)]


class rc_norm(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("C", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("post", ctypes.c_int32), ("N", ctypes.c_int64), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float), ("mod_batch", ctypes.c_int64), ("mod_group", ctypes.c_int64),
                ("n_spans", ctypes.c_int32), ("rows", ctypes.c_int32 * RC_MAX_SEGMENTS),
                ("group", ctypes.c_int32 * RC_MAX_SEGMENTS)]


_LIB = None
_vp, _i32, _i64, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_f64 = ctypes.c_double
_PL, _PR, _PN = ctypes.POINTER(rc_layout), ctypes.POINTER(rc_rotary), ctypes.POINTER(rc_norm)
_PB = ctypes.POINTER(rc_blocks8)
SIGNATURES = {
    "rc_layout_preset": (_i32, [_PL, _i32]),
    "rc_layout_validate": (_i32, [_PL, _i32]),
    "rc_pairs": (_i64, [_PL, _i32]),
    "rc_rows": (_i64, [_PL, _i32]),
    "rc_step_workspace_bytes": (_sz, [_PL, _i32, _i32, _i32, _i32]),
    "rc_step_auto_splits": (_i32, [_PL, _i32, _i32, _i32]),
    "rc_ref_kv_prefill": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp]),
    "rc_step_masked_attention": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp,
                                        _i32, _vp, _sz, _vp]),
    "rc_full_attention": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp]),
    "rc_linear": (_i32, [_i64, _i32, _i32, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp]),
    "rc_ref_kv_prefill_fp8": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp,
                                     _vp]),
    "rc_step_masked_attention_fp8": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp,
                                            _vp, _i32, _vp, _sz, _vp]),
    "rc_step_masked_attention_noalloc": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp,
                                                _vp, _i32, _vp]),
    "rc_step_launch_shape": (_i32, [_PL, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(_i64),
                                    ctypes.POINTER(_i32), ctypes.POINTER(_i32)]),
    "rc_attention_work_groups": (_i64, [_PL, _i32, _i32, _i32, _i32, _i32, _i32]),
    "rc_full_attention_ws": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "rc_full_workspace_bytes": (_sz, [_PL, _i32, _i32, _i32]),
    "rc_prefill_launch_plan": (_i32, [_PL, _i32, _i32, _i32, ctypes.POINTER(_i64), ctypes.POINTER(_i32),
                                      ctypes.POINTER(_i64)]),
    "rc_full_backward_workspace_bytes": (_sz, [_PL, _i32, _i32, _i32]),
    "rc_full_attention_backward": (_i32, [_PL, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp,
                                          _vp, _vp, _i64, _vp, _sz, _vp]),
    "rc_rotary_init": (_i32, [_PR, _i32, _i32, ctypes.POINTER(_i32), _f64, _i32, _i32]),
    "rc_qk_rotary": (_i32, [_PR, _i32, _i64, _i32, _vp, _vp, _i64, _vp, _i32, _i32, _vp, _vp, _f32, _vp, _vp, _i64,
                            _vp]),
    "rc_rotary_backward_workspace_bytes": (_sz, [_PR, _i32, _i64]),
    "rc_qk_rotary_backward": (_i32, [_PR, _i32, _i64, _i32, _vp, _vp, _i64, _vp, _i32, _i32, _vp, _vp, _i64, _vp, _vp,
                                     _f32, _vp, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "rc_gated_norm": (_i32, [_PN, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "rc_gated_norm_backward_workspace_bytes": (_sz, [_PN]),
    "rc_gated_norm_backward": (_i32, [_PN, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64,
                                      _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "rc_quantize_blocks": (_i32, [_i64, _i32, _vp, _i64, _i32, _PB, _PB, _vp]),
    "rc_dequantize_blocks": (_i32, [_i64, _i32, _PB, _vp, _i64, _vp]),
    "rc_linear_fp8_blocks": (_i32, [_i64, _i32, _i32, _PB, _PB, _vp, _i64, _vp, _i64, _vp]),
    "rc_linear_fp8": (_i32, [_i64, _i32, _i32, _vp, _i64, _PB, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "rc_linear_fp8_workspace_bytes": (_sz, [_i64, _i32, _i32]),
    "rc_linear_fp8_backward": (_i32, [_i64, _i32, _i32, _vp, _i64, _PB, _PB, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _sz,
                                      _vp]),
    "rc_linear_fp8_backward_workspace_bytes": (_sz, [_i64, _i32, _i32, _i32, _i32]),
    "rc_status_string": (ctypes.c_char_p, [_i32]),
    "rc_last_error": (ctypes.c_char_p, []),
}


def lib():
    """The loaded library; raises if it was not built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_21229_amd.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


def _check(status: int):
    if status != RC_OK:
        raise RcError(status, lib().rc_last_error().decode())


class Layout:
    """Segment table + block mask (rc_layout).

    segments: (kind, length) pairs in sequence order, kinds SEG_*.
    mask: a preset name ('paper', 'perref', 'isolated', 'dense'), a MASK_*
    id, or an explicit query-first boolean matrix over segments.
    """

    def __init__(self, segments: Sequence[Tuple[int, int]], mask="perref"):
        if not 1 <= len(segments) <= RC_MAX_SEGMENTS:
            raise ValueError(f"need 1..{RC_MAX_SEGMENTS} segments")
        self.c = rc_layout()
        self.c.n_seg = len(segments)
        for i, (k, n) in enumerate(segments):
            self.c.seg[i].kind = int(k)
            self.c.seg[i].len = int(n)
        self.segments = [(int(k), int(n)) for k, n in segments]
        if isinstance(mask, str) or isinstance(mask, int):
            preset = MASKS[mask] if isinstance(mask, str) else mask
            _check(lib().rc_layout_preset(ctypes.byref(self.c), preset))
        else:
            for q, row in enumerate(mask):
                self.c.visible[q] = sum(1 << k for k, v in enumerate(row) if v)

    @property
    def visible(self):
        n = self.c.n_seg
        return [[bool(self.c.visible[q] >> k & 1) for k in range(n)] for q in range(n)]

    def validate(self, entry: int) -> int:
        return lib().rc_layout_validate(ctypes.byref(self.c), entry)

    def pairs(self, entry: int) -> int:
        v = lib().rc_pairs(ctypes.byref(self.c), entry)
        if v < 0:
            _check(int(v))
        return int(v)

    def rows(self, which: int) -> int:
        v = lib().rc_rows(ctypes.byref(self.c), which)
        if v < 0:
            _check(int(v))
        return int(v)

    def workspace_bytes(self, B: int, H: int, D: int, splits: int = 0) -> int:
        return int(lib().rc_step_workspace_bytes(ctypes.byref(self.c), B, H, D, splits))

    def launch_shape(self, B: int, H: int, D: int, splits: int = 0, fp8: bool = False):
        """(work-groups, query rows per work-group, resolved splits) of the
        step's attention kernel, a tile run as two halves counted once
        (``work_groups`` counts what is launched)."""
        wg, bm, sp = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib().rc_step_launch_shape(ctypes.byref(self.c), B, H, D, splits, int(fp8), ctypes.byref(wg),
                                          ctypes.byref(bm), ctypes.byref(sp)))
        return wg.value, bm.value, sp.value

    def work_groups(self, entry: int, B: int, H: int, D: int, splits: int = 1, fp8: bool = False) -> int:
        """Work-groups that an attention call launches (ENTRY_*), tiles run as
        two halves counted twice; see rc_attention_work_groups."""
        n = lib().rc_attention_work_groups(ctypes.byref(self.c), entry, B, H, D, splits, int(fp8))
        if n < 0:
            _check(int(n))
        return int(n)

    def full_workspace_bytes(self, B: int, H: int, D: int) -> int:
        """Workspace of the full recompute's last-round split (0: no split)."""
        return int(lib().rc_full_workspace_bytes(ctypes.byref(self.c), B, H, D))

    def backward_workspace_bytes(self, B: int, H: int, D: int) -> int:
        """Workspace of the full recompute's gradient."""
        return int(lib().rc_full_backward_workspace_bytes(ctypes.byref(self.c), B, H, D))

    def prefill_plan(self, B: int, H: int, D: int):
        """(attention work-groups, copy work-groups, cache rows they copy) of
        the bf16 prefill; the store kernel copies the remaining rows."""
        a, c, r = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int64()
        _check(lib().rc_prefill_launch_plan(ctypes.byref(self.c), B, H, D, ctypes.byref(a), ctypes.byref(c),
                                            ctypes.byref(r)))
        return a.value, c.value, r.value

    def modulation_spans(self, which: int = ROWS_ALL, live: int = 0, static: int = 1):
        """(rows, group) spans of a row class for gated_norm: live segments
        (text, target) take group `live`, static ones (anchors, references) `static`."""
        if which not in (ROWS_STATIC, ROWS_LIVE, ROWS_ALL):
            raise ValueError(f"modulation spans are those of ROWS_STATIC, ROWS_LIVE or ROWS_ALL, got {which!r}")
        spans = []
        for k, n in self.segments:
            is_live = k in (SEG_TEXT, SEG_TARGET)
            if which == ROWS_ALL or (which == ROWS_LIVE) == is_live:
                spans.append((n, live if is_live else static))
        return spans

    def auto_splits(self, B: int, H: int, D: int) -> int:
        return int(lib().rc_step_auto_splits(ctypes.byref(self.c), B, H, D))


# ---------------------------------------------------------------- tensor entry points
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _tok_stride(*ts) -> int:
    st = ts[0].stride()
    B, N, H, D = ts[0].shape
    if st[3] == 1 and st[2] == D and (B == 1 or st[0] == N * st[1]) and all(t.stride() == st for t in ts[1:]):
        return st[1]  # one shape (checked before) and one layout
    strides = set()
    for t in ts:
        B, N, H, D = t.shape
        if t.stride(3) != 1 or t.stride(2) != D or (B > 1 and N > 1 and t.stride(0) != N * t.stride(1)):
            raise ValueError("Q/K/V must be [B, N, H, D] with D contiguous, head stride D and batch stride N*tok_stride")
        # of one token the batch stride is the token stride; no token, or one of one entry, is at any stride
        strides.add(t.stride(1) if N > 1 else t.stride(0) if N == 1 and B > 1 else H * D)
    if len(strides) != 1:
        raise ValueError("Q, K and V must share one token stride")
    return strides.pop()


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _expect(t, shape, dtype_name, what):
    """Outputs and the cache use the library's contiguous layouts."""
    if t is None or (t.shape == shape and t.is_contiguous() and str(t.dtype) == dtype_name):
        return
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous() or str(t.dtype) != dtype_name:
        raise ValueError(f"{what} must be a contiguous {dtype_name} tensor of shape {tuple(shape)}, "
                         f"got {str(t.dtype)} {tuple(t.shape)} contiguous={t.is_contiguous()}")


def _call(fn, dev, stream, *args):
    """fn(*args, stream) with dev as the current device and the handle of its
    current stream where none is given.

    Looking up the stream object (2.0 us) and entering and leaving the device
    (2.3 us) cost more than the rest of a small call, so the raw handle is
    asked for and the device only entered where it is not current.  With the
    tensor checks' first tests below, a projection of 16 rows takes the host
    7.1 us instead of 10.7, a tiny step 11.6 instead of 16.5."""
    torch = _torch()
    if torch.cuda.current_device() != dev.index:
        with torch.cuda.device(dev):
            return _call(fn, dev, stream, *args)
    _check(fn(*args, torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream))


def _on(stream, dev):
    """Context in which the caller's stream is the current one."""
    cuda = _torch().cuda
    return cuda.stream(stream if isinstance(stream, cuda.Stream)
                       else cuda.ExternalStream(stream.cuda_stream, device=dev))


def _empty(shape, dtype, dev, stream, returned=True):
    """Memory that a call allocates for itself.  With a stream given it is that
    stream's: memory of the current stream would be free for the current
    stream's next allocation as soon as its tensor is dropped (a workspace: on
    return), while the call's kernels still use it.  A returned tensor is
    marked as used on the current stream too, where the caller reads it."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with _on(stream, dev):
        t = torch.empty(shape, dtype=dtype, device=dev)
    if returned:
        t.record_stream(torch.cuda.current_stream(dev))
    return t


def _like(t, dev, stream):
    """A contiguous tensor of t's shape and type, allocated as by _empty.  A
    small call's time is mostly the host's: empty_like takes 1.2 us, empty with
    a shape, type and device 1.7, with the shape still a tensor's 2.2."""
    if stream is None and t.is_contiguous():
        return _torch().empty_like(t)
    return _empty(tuple(t.shape), t.dtype, dev, stream)


def _inputs(q, k, v):
    """Q/K/V: bf16 tensors of one shape on one GPU; returns that device.  The
    library takes raw device pointers, so a host tensor must never reach it."""
    dev = q.device
    bf16, shape = _torch().bfloat16, q.shape
    if (q.is_cuda and q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and k.shape == shape
            and v.shape == shape and k.device == dev and v.device == dev):
        return dev
    if dev.type != "cuda":
        raise ValueError(f"q must be a GPU tensor, got device {dev}")
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.device != dev or str(t.dtype) != "torch.bfloat16" or tuple(t.shape) != tuple(q.shape):
            raise ValueError(f"{name} must be a bf16 tensor of shape {tuple(q.shape)} on {dev}, "
                             f"got {str(t.dtype)} {tuple(t.shape)} on {t.device}")
    return dev


def _rows_of(layout: "Layout", q, which: int, what: str):
    """The library sizes every read and write from the layout's row count, so
    Q must hold exactly that many tokens (checked before anything else)."""
    n = layout.rows(which)
    if q.dim() != 4 or q.shape[1] != n:
        raise ValueError(f"{what}: q must be [B, {n}, H, D] (the layout's row count), got {tuple(q.shape)}")


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the inputs on {dev}")


def ref_kv_prefill(layout: Layout, q, k, v, o=None, lse=None, k_cache=None, v_cache=None,
                   scale: Optional[float] = None, want_lse: bool = False, stream=None):
    """Static-subgraph prefill.  q/k/v: [B, N_static, H, D] bf16 (ST and R
    tokens in sequence order).  Returns (o, lse or None, k_cache, v_cache)."""
    torch = _torch()
    _rows_of(layout, q, ROWS_STATIC, "ref_kv_prefill")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    nc = layout.rows(ROWS_CACHED)
    if o is None:
        o = _empty((B, N, H, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _empty((B, H, N), torch.float32, dev, stream)
    if k_cache is None:
        k_cache = _empty((B, H, nc, D), torch.bfloat16, dev, stream)
    if v_cache is None:
        v_cache = _empty((B, H, nc, D), torch.bfloat16, dev, stream)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(k_cache, (B, H, nc, D), "torch.bfloat16", "k_cache")
    _expect(v_cache, (B, H, nc, D), "torch.bfloat16", "v_cache")
    _same_device(dev, o=o, lse=lse, k_cache=k_cache, v_cache=v_cache)
    _call(lib().rc_ref_kv_prefill, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(), k.data_ptr(),
          v.data_ptr(), ts, o.data_ptr(), _ptr(lse), k_cache.data_ptr(), v_cache.data_ptr())
    return o, lse, k_cache, v_cache


def step_masked_attention(layout: Layout, q, k, v, k_cache, v_cache, o=None, lse=None, splits: int = 0,
                          workspace=None, scale: Optional[float] = None, want_lse: bool = False, stream=None):
    """Per-step attention.  q/k/v: [B, N_live, H, D] bf16 (LT and X tokens);
    k_cache/v_cache: [B, H, N_cached, D].  splits: 0 automatic, 1 none, > 1
    even split-KV, SPLITS_TAIL the tail split, SPLITS_LAST_ROUND the tail split
    of the last round's tiles, SPLITS_BALANCED the balanced schedule.  Returns
    (o, lse or None)."""
    torch = _torch()
    _rows_of(layout, q, ROWS_LIVE, "step_masked_attention")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    if o is None:
        o = _empty((B, N, H, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _empty((B, H, N), torch.float32, dev, stream)
    nc = layout.rows(ROWS_CACHED)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(k_cache, (B, H, nc, D), "torch.bfloat16", "k_cache")
    _expect(v_cache, (B, H, nc, D), "torch.bfloat16", "v_cache")
    need = layout.workspace_bytes(B, H, D, splits)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _empty(need, torch.uint8, dev, stream, returned=False)
    _same_device(dev, o=o, lse=lse, k_cache=k_cache, v_cache=v_cache, workspace=workspace if need else None)
    _call(lib().rc_step_masked_attention, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(),
          k.data_ptr(), v.data_ptr(), ts, _ptr(k_cache), _ptr(v_cache), o.data_ptr(), _ptr(lse), splits,
          _ptr(workspace) if need else None, need)
    return o, lse


def step_masked_attention_noalloc(layout: Layout, q, k, v, k_cache, v_cache, o, lse=None, splits: int = 0,
                                  scale: Optional[float] = None, stream=None):
    """step_masked_attention without any device allocation: the caller passes
    the output `o` (and `lse`, or None), and split partials go to the
    library's static scratch array (NOALLOC_SCRATCH_BYTES per GPU; a larger
    split choice raises RcError with RC_ERR_WORKSPACE).  Calls that overlap on
    one GPU share that array and race.  Returns (o, lse)."""
    if o is None:
        raise ValueError("step_masked_attention_noalloc: pass the output o (it allocates nothing)")
    _rows_of(layout, q, ROWS_LIVE, "step_masked_attention_noalloc")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    nc = layout.rows(ROWS_CACHED)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(k_cache, (B, H, nc, D), "torch.bfloat16", "k_cache")
    _expect(v_cache, (B, H, nc, D), "torch.bfloat16", "v_cache")
    _same_device(dev, o=o, lse=lse, k_cache=k_cache, v_cache=v_cache)
    _call(lib().rc_step_masked_attention_noalloc, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(),
          k.data_ptr(), v.data_ptr(), ts, _ptr(k_cache), _ptr(v_cache), o.data_ptr(), _ptr(lse), splits)
    return o, lse


def full_attention(layout: Layout, q, k, v, o=None, lse=None, scale: Optional[float] = None,
                   want_lse: bool = False, last_round_split: bool = True, stream=None):
    """Full recompute over all rows.  q/k/v: [B, N, H, D] bf16.  Returns (o, lse or None).
    last_round_split: give the library the workspace it asks for to split the
    grid's partial last round (rc_full_attention_ws); False computes every
    query tile whole (rc_full_attention)."""
    torch = _torch()
    _rows_of(layout, q, ROWS_ALL, "full_attention")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    if o is None:
        o = _empty((B, N, H, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _empty((B, H, N), torch.float32, dev, stream)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _same_device(dev, o=o, lse=lse)
    need = layout.full_workspace_bytes(B, H, D) if last_round_split else 0
    ws = _empty(need, torch.uint8, dev, stream, returned=False) if need else None
    _call(lib().rc_full_attention_ws, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(), k.data_ptr(),
          v.data_ptr(), ts, o.data_ptr(), _ptr(lse), _ptr(ws), need)
    return o, lse


def full_attention_backward(layout: Layout, q, k, v, o, lse, do, dq=None, dk=None, dv=None, dlse=None,
                            scale: Optional[float] = None, workspace=None, stream=None):
    """Gradient of full_attention.  q/k/v, o and lse: the forward's inputs and
    outputs (want_lse=True); do, dlse (None: zero): the gradients of o and
    lse.  dq, dk and dv share one token stride (views of one [B, N, 3, H, D]
    buffer work) and overlap no input.  Returns (dq, dk, dv), bf16."""
    torch = _torch()
    _rows_of(layout, q, ROWS_ALL, "full_attention_backward")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    if o is None or lse is None or do is None:
        raise ValueError("full_attention_backward: pass the forward's o and lse (want_lse=True) and do")
    grads, gs = [dq, dk, dv], H * D
    if dq is None and dk is None and dv is None:
        first = _like(q, dev, stream)
        grads = [first, _like(first, dev, stream), _like(first, dev, stream)]
    else:
        grads = [g if g is not None else _like(q, dev, stream) for g in grads]
        for name, t in zip(("dq", "dk", "dv"), grads):
            if t.dtype is not torch.bfloat16 or t.shape != q.shape:
                raise ValueError(f"{name} must be a bf16 tensor of shape {tuple(q.shape)}, got {str(t.dtype)} "
                                 f"{tuple(t.shape)}")
        gs = _tok_stride(*grads)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(do, (B, N, H, D), "torch.bfloat16", "do")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(dlse, (B, H, N), "torch.float32", "dlse")
    mine = workspace
    need = layout.backward_workspace_bytes(B, H, D)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = _empty(need, torch.uint8, dev, stream, returned=False)
    if not (o.device == dev and do.device == dev and lse.device == dev and dlse is None and mine is None
            and dq is None and dk is None and dv is None):
        _same_device(dev, o=o, do=do, lse=lse, dlse=dlse, dq=grads[0], dk=grads[1], dv=grads[2], workspace=mine)
    _call(lib().rc_full_attention_backward, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(),
          k.data_ptr(), v.data_ptr(), ts, o.data_ptr(), lse.data_ptr(), do.data_ptr(), _ptr(dlse), grads[0].data_ptr(),
          grads[1].data_ptr(), grads[2].data_ptr(), gs, workspace.data_ptr(), need)
    return tuple(grads)


def _rows_view(t, what):
    """A [M, n] bf16 GPU view with unit column stride; returns its row stride."""
    if t.dim() != 2 or t.dtype is not _torch().bfloat16 or not t.is_cuda:
        raise ValueError(f"{what} must be a 2-D bf16 GPU tensor, got {str(t.dtype)} {tuple(t.shape)} on {t.device}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must have unit column stride")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def linear(a, w, residual=None, out=None, stream=None):
    """out = a @ w.T (+ residual), bf16 in and out, fp32 accumulation.
    a: [M, K] (any row stride); w: [N, K] contiguous; residual, out: [M, N]
    (any row stride; out may be residual).  Returns out."""
    torch = _torch()
    lda = _rows_view(a, "a")
    dev = a.device
    M, K = a.shape
    if w.dim() != 2 or w.shape[1] != K or not w.is_contiguous() or w.dtype is not torch.bfloat16:
        raise ValueError(f"w must be a contiguous bf16 [N, {K}] tensor, got {str(w.dtype)} {tuple(w.shape)}")
    N = w.shape[0]
    if out is None:
        out = _empty((M, N), torch.bfloat16, dev, stream)
    for name, t in (("out", out), ("residual", residual)):
        if t is not None and t.shape != (M, N):
            raise ValueError(f"{name} must have shape {(M, N)}, got {tuple(t.shape)}")
    ldo = _rows_view(out, "out")
    ldr = _rows_view(residual, "residual") if residual is not None else 0
    _same_device(dev, w=w, out=out, residual=residual)
    _call(lib().rc_linear, dev, stream, M, N, K, a.data_ptr(), lda, w.data_ptr(), _ptr(residual), ldr, out.data_ptr(),
          ldo)
    return out


# ---------------------------------------------------------------- projections in 8 bits
class Fp8Blocks:
    """A [rows, cols] matrix as e4m3 codes with one power-of-two scale per block
    of 128 values (rc_blocks8), made by ``quantize_blocks``.

    codes: uint8 [rows, cols rounded up to 128], zeros past the last column;
    exps: uint8 [blocks of a row, rows rounded up to 16], exponent + 127 of the
    block of (row, col) at [col // 128, row]; t: the transposed matrix, for
    weights quantised with ``transposed=True``, else None."""

    __slots__ = ("codes", "exps", "shape", "t", "c", "device")

    def __init__(self, codes, exps, shape, t=None):
        rows, cols = shape
        want = (rows, -(-cols // 128) * 128), (-(-cols // 128), -(-rows // 16) * 16)
        for x, w, what in ((codes, want[0], "codes"), (exps, want[1], "exps")):
            _expect(x, w, "torch.uint8", what)
        _same_device(codes.device, exps=exps, t=t)
        if t is not None and t.shape != (cols, rows):
            raise ValueError(f"t must be {(cols, rows)}, got {t.shape}")
        self._set(codes, exps, (rows, cols), t)

    def _set(self, codes, exps, shape, t):
        self.codes, self.exps, self.shape, self.t, self.device = codes, exps, shape, t, codes.device
        self.c = rc_blocks8(codes.data_ptr(), -(-shape[1] // 128) * 128, exps.data_ptr(), -(-shape[0] // 16) * 16)

    @staticmethod
    def empty(rows, cols, device, stream=None, t=None):
        """Memory for [rows, cols] (of stream's, as a call's own outputs)."""
        u8, blocks = _torch().uint8, -(-cols // 128)
        b = Fp8Blocks.__new__(Fp8Blocks)
        b._set(_empty((rows, blocks * 128), u8, device, stream), _empty((blocks, -(-rows // 16) * 16), u8, device, stream),
               (rows, cols), t)
        return b


def _blocks(b, what, rows=None, cols=None):
    """Checked Fp8Blocks on a GPU; their shape."""
    if not isinstance(b, Fp8Blocks):
        raise ValueError(f"{what} must be Fp8Blocks (quantize_blocks makes them), got {type(b).__name__}")
    if b.device.type != "cuda":
        raise ValueError(f"{what} must be on a GPU, got {b.device}")
    m, k = b.shape
    if (rows is not None and m != rows) or (cols is not None and k != cols):
        raise ValueError(f"{what} must be {(m if rows is None else rows, k if cols is None else cols)}, got {(m, k)}")
    return m, k


def quantize_blocks(x, square=False, transposed=False, out=None, stream=None) -> Fp8Blocks:
    """x [M, K] bf16 (any row stride) in e4m3 with one power-of-two scale per
    128 values of a row, or with ``square`` per 128 x 128 values; ``transposed``
    (square only): with the transposed matrix as ``.t``, which the inputs'
    gradient of a projection reads.  Weights are quantised once, square; activations per
    call, and what a projection has read is the checkpoint for its weights' gradient."""
    ldx = _rows_view(x, "x")
    dev = x.device
    M, K = x.shape
    if transposed and not square:
        raise ValueError("transposed needs square=True: a block of a row is no block of its transpose")
    if out is None:
        out = Fp8Blocks.empty(M, K, dev, stream, Fp8Blocks.empty(K, M, dev, stream) if transposed else None)
    else:
        _blocks(out, "out", M, K)
        if transposed:
            _blocks(out.t, "out.t", K, M)
        elif out.t is not None:
            raise ValueError("out has a transposed form, which would stay what it is: transposed=True, or another out")
        _same_device(dev, out=out)
        _apart_from(out, "out", x=x)
        if transposed:
            _apart_from(out.t, "out.t", x=x, out=out)
    _call(lib().rc_quantize_blocks, dev, stream, M, K, x.data_ptr(), ldx, int(square), ctypes.byref(out.c),
          ctypes.byref(out.t.c) if transposed else None)
    return out


def dequantize_blocks(x, out=None, stream=None):
    """The values of Fp8Blocks in bf16 [M, K] (exact below 2^128, infinite there).  Returns out."""
    M, K = _blocks(x, "x")
    dev, given = x.device, out is not None
    out, ldo = _rows_out(out, "out", M, K, dev, stream)
    if given:
        _apart_from(out, "out", x=x)
    _call(lib().rc_dequantize_blocks, dev, stream, M, K, ctypes.byref(x.c), out.data_ptr(), ldo)
    return out


def linear_fp8(a, w, residual=None, out=None, workspace=None, stream=None):
    """out = a @ w.T (+ residual) in 8 bits: w [N, K] Fp8Blocks, a [M, K] Fp8Blocks
    or bf16 (any row stride; quantised per 128 values of a row on the way, into the
    workspace); bf16 out, summed in fp32 of products that are cut, towards zero, below
    2^-13 of the largest power of two among eight neighbouring ones (as
    rc_linear_fp8_blocks says).  residual, out: [M, N] (any row
    stride; out may be residual as it lies).  What is given to write to (out, workspace) may lie
    beside the inputs in one buffer, but shares no memory with them.  A row's result does not depend on M for
    Fp8Blocks; a small bf16 call (up to 32 rows, or little work) sums in another order.
    Returns out."""
    L, blocks = lib(), isinstance(a, Fp8Blocks)
    lda = 0 if blocks else _rows_view(a, "a")
    M, K = _blocks(a, "a") if blocks else a.shape
    dev, N = a.device, _blocks(w, "w", cols=K)[0]
    given = out is not None
    out, ldo = _rows_out(out, "out", M, N, dev, stream)
    ldr = _rows_in(residual, "residual", M, N, dev)
    if given:
        _apart(out, "out", ldo, None if blocks else a, "a", residual, ldr)
        _apart_from(out, "out", a=a if blocks else None, w=w)
    if w.device != dev:
        raise ValueError(f"w is on {w.device}, the inputs on {dev}")
    if blocks:
        _call(L.rc_linear_fp8_blocks, dev, stream, M, N, K, ctypes.byref(a.c), ctypes.byref(w.c), _ptr(residual), ldr,
              out.data_ptr(), ldo)
        return out
    need = L.rc_linear_fp8_workspace_bytes(M, N, K)
    workspace, own = (_workspace(workspace, need, dev, stream) if need else None), workspace
    if need and workspace is own:
        _apart_from((_place(own.data_ptr(), need, need, 1),), "workspace", a=a, w=w, residual=residual, out=out)
    _call(L.rc_linear_fp8, dev, stream, M, N, K, a.data_ptr(), lda, ctypes.byref(w.c), _ptr(residual), ldr,
          out.data_ptr(), ldo, _ptr(workspace), need)
    return out


def _rows_out(t, what, rows, cols, dev, stream):
    """A bf16 output [rows, cols] and its row stride: the caller's, or new memory, which needs no checks."""
    if t is None:
        return _empty((rows, cols), _torch().bfloat16, dev, stream), cols
    return t, _rows_in(t, what, rows, cols, dev)


def _apart(out, what, ldo, a, name, residual, ldr):
    """Refuses the caller's output where it shares memory with the input a (None: no bf16 one), or with the
    residual other than as it lies."""
    at, r = out.data_ptr(), None if residual is None else residual.data_ptr()
    if a is None and (r is None or (r == at and ldr == ldo)):
        return
    n, w = out.shape
    if not n or not w:
        return
    end = at + 2 * ((n - 1) * ldo + w)
    if a is not None and a.data_ptr() < end and _meet(_rows_at(out), _rows_at(a)):
        raise ValueError(f"{what} may not be {name}, which is read while it is written, nor overlap it")
    if r is None:
        return
    if r == at and ldr != ldo:
        raise ValueError(f"{what} may be residual only with its row stride, {ldr}, got {ldo}")
    if r != at and r < end and at < r + 2 * ((n - 1) * ldr + w) and _meet(_rows_at(out), _rows_at(residual)):
        raise ValueError(f"{what} may be residual as it lies, but not overlap it otherwise")


def _apart_from(t, what, **others):
    """Refuses a caller's output (a tensor or Fp8Blocks) or a workspace's place that shares memory with
    others, None where absent, which the call reads or writes too."""
    mine = t if type(t) is tuple else _places(t)
    for name, o in others.items():
        if o is None:
            continue
        for b in _places(o):
            for a in mine:
                if b[0] < a[4] and a[0] < b[4] and _meet(a, b):
                    raise ValueError(f"{what} may not overlap {name}")


def _place(p, width, stride, rows):
    return p, width, stride, rows, p + (rows - 1) * stride + width


def _rows_at(t):
    """Where a tensor lies: its first byte, the bytes of a row, those from one row to the next, the rows, and
    where it ends.  One that is no matrix is contiguous here: one row."""
    p = t.data_ptr()
    if t.is_contiguous():
        n = t.nbytes
        return p, n, n, 1, p + n
    size = t.itemsize
    return _place(p, t.shape[1] * size, t.stride(0) * size, t.shape[0])


def _places(t):
    """The same of all that a tensor or Fp8Blocks (without their transposed form) hold."""
    if not isinstance(t, Fp8Blocks):
        return (_rows_at(t),)
    c, (rows, cols) = t.c, t.shape
    n, m, p, q = rows * c.ld, -(-cols // 128) * c.ld_exps, c.codes or 0, c.exps or 0
    return (p, n, n, 1, p + n), (q, m, m, 1, q + m)


def _meet(a, b):
    """Whether two places of _rows_at share a byte: their ranges do, and they are not columns side by
    side, which stay apart in every row where they do in one (modulo what divides both strides)."""
    (p, w, s, n, end), (q, v, u, m, ends) = a, b
    if not (n and m and w and v) or end <= q or ends <= p:
        return False
    g = math.gcd(s if n > 1 else 0, u if m > 1 else 0)
    r = (q - p) % g if g else 0
    return not (w <= r <= g - v)


def _rows_in(t, what, rows, cols, dev):
    """The row stride of a checked bf16 [rows, cols] tensor; 0 for None."""
    if t is None:
        return 0
    if t.shape != (rows, cols):
        raise ValueError(f"{what} must have shape {(rows, cols)}, got {tuple(t.shape)}")
    ld = _rows_view(t, what)
    if t.device != dev:
        raise ValueError(f"{what} is on {t.device}, the inputs on {dev}")
    return ld


def linear_fp8_backward(dy, x, w, residual=None, dx=None, dw=None, want_dx=True, want_dw=True, workspace=None,
                        stream=None):
    """The gradient of linear_fp8 for dy [M, N] bf16: x [M, K] Fp8Blocks, the input
    that the product has read; w [N, K] Fp8Blocks with their transposed form.
    dx [M, K] bf16 = dy @ w (+ residual), dy quantised per 128 values of a row, its
    products cut as linear_fp8's;
    dw [N, K] fp32 = dy.T @ x with dy as it is and x as dequantize_blocks expands it.  dx may be residual as it lies; otherwise dx,
    dw and workspace share no memory with the inputs or each other.  A workspace serves one
    call at a time.  Returns (dx, dw), None for what is not wanted (x and w may then be None)."""
    L, lddy, lddx, ldr, w_t = lib(), _rows_view(dy, "dy"), 0, 0, None
    dev = dy.device
    M, N = dy.shape
    if not (want_dx or want_dw):
        raise ValueError("neither dx nor dw is wanted")
    if residual is not None and not want_dx:
        raise ValueError("residual goes with dx")
    if (dx is not None and not want_dx) or (dw is not None and not want_dw):
        raise ValueError("dx or dw is given but not wanted")
    K = (_blocks(w, "w", rows=N) if want_dx else _blocks(x, "x", rows=M))[1]
    if want_dw:
        _blocks(x, "x", M, K)
    if want_dx:
        w_t = w.t
        if w_t is None:
            raise ValueError("w has no transposed form: quantize_blocks(w, square=True, transposed=True)")
        _blocks(w_t, "w.t", K, N)
        given = dx is not None
        dx, lddx = _rows_out(dx, "dx", M, K, dev, stream)
        ldr = _rows_in(residual, "residual", M, K, dev)
        if given:
            _apart(dx, "dx", lddx, dy, "dy", residual, ldr)
            _apart_from(dx, "dx", w=w_t, x=x if want_dw else None)
    if want_dw:
        if dw is None:
            dw = _empty((N, K), _torch().float32, dev, stream)
        else:
            _expect(dw, (N, K), "torch.float32", "dw")
            _same_device(dev, dw=dw)
            _apart_from(dw, "dw", dy=dy, x=x, w=w_t, residual=residual, dx=dx)
    _same_device(dev, x=x if want_dw else None, w=w_t)
    need = L.rc_linear_fp8_backward_workspace_bytes(M, N, K, int(want_dx), int(want_dw))
    workspace, own = (_workspace(workspace, need, dev, stream) if need else None), workspace
    if need and workspace is own:
        _apart_from((_place(own.data_ptr(), need, need, 1),), "workspace", dy=dy, x=x if want_dw else None, w=w_t,
                    residual=residual, dx=dx, dw=dw)
    _call(L.rc_linear_fp8_backward, dev, stream, M, N, K, dy.data_ptr(), lddy, ctypes.byref(x.c) if want_dw else None,
          ctypes.byref(w_t.c) if want_dx else None, _ptr(residual), ldr, _ptr(dx), lddx, _ptr(dw), K, _ptr(workspace), need)
    return dx, dw


def _workspace(workspace, need, dev, stream):
    """The caller's workspace where it is large enough, else one of this call's."""
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        return _empty(need, _torch().uint8, dev, stream, returned=False)
    _same_device(dev, workspace=workspace)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace


# ---------------------------------------------------------------- rotation of queries and keys
class Rotary:
    """How a head row's channels turn with the token's position (rc_rotary).

    axes: rotated widths per position axis, e.g. (16, 56, 56) for (time,
    height, width) of 128-wide heads; channels past their sum stay.
    interleaved: pairs of neighbouring channels, else of the rotated width's
    two halves.  continuous: one frequency ladder over all axes, else each
    axis has its own from 1 down to 1 / theta."""

    def __init__(self, head_dim: int, axes: Sequence[int], theta: float = 10000.0, interleaved: bool = True,
                 continuous: bool = False):
        self.c = rc_rotary()
        self.head_dim, self.axes = int(head_dim), tuple(int(a) for a in axes)
        arr = (ctypes.c_int32 * max(1, len(self.axes)))(*self.axes)
        _check(lib().rc_rotary_init(ctypes.byref(self.c), self.head_dim, len(self.axes), arr, float(theta),
                                    int(interleaved), int(continuous)))


def _heads(name, t, like=None, D=None):
    """A bf16 [B, N, H, D] GPU tensor, of like's shape and device."""
    if t.dim() != 4 or t.dtype is not _torch().bfloat16 or not t.is_cuda or (D is not None and t.shape[3] != D):
        raise ValueError(f"{name} must be a bf16 [B, N, H, {D or 'D'}] GPU tensor, got {str(t.dtype)} "
                         f"{tuple(t.shape)} on {t.device}")
    if like is not None and (t.shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must have shape {tuple(like.shape)} on {like.device}, got {tuple(t.shape)} on {t.device}")


def _given(*ts):
    return [t for t in ts if t is not None]


def _pair(names, q, k, D):
    """The tensors given of a pair of queries and keys, checked: bf16
    [B, N, H, D] on one GPU.  The first test covers the usual call."""
    if q is not None and k is not None:
        bf16 = _torch().bfloat16
        if (q.dtype is bf16 and k.dtype is bf16 and q.is_cuda and q.device == k.device and q.shape == k.shape
                and q.dim() == 4 and q.shape[3] == D):
            return [q, k]
    given = _given(q, k)
    if not given:
        raise ValueError(f"pass {names[0]}, {names[1]} or both")
    for name, t in zip(names, (q, k)):
        if t is not None:
            _heads(name, t, given[0], D)
    return given


def _positions(rotary: Rotary, t, positions):
    """(is fp32, has a batch axis) of the positions of t's tokens."""
    torch = _torch()
    floats, shape, batch = positions.dtype is torch.float32, positions.shape, positions.dim() == 3
    if not (floats or positions.dtype is torch.int32) or not positions.is_contiguous():
        raise ValueError(f"positions must be contiguous int32 or float32, got {str(positions.dtype)}")
    B, N, A = t.shape[0], t.shape[1], len(rotary.axes)
    if shape != ((B, N, A) if batch else (N, A)):
        raise ValueError(f"positions must be {(N, A)} or {(B, N, A)}, got {tuple(shape)}")
    return int(floats), int(batch)


def _norm_weight(name, w, D):
    if w is not None and (w.dtype is not _torch().bfloat16 or tuple(w.shape) != (D,) or not w.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous bf16 [{D}] tensor, got {str(w.dtype)} {tuple(w.shape)}")


def _outputs(outs, ins, names, dev, stream):
    """An output per input (None where there is none), and their token stride."""
    if outs[0] is None and outs[1] is None:
        shape = (ins[0] if ins[0] is not None else ins[1]).shape
        first = _like(ins[0] if ins[0] is not None else ins[1], dev, stream)
        if ins[0] is None or ins[1] is None:
            return [None if i is None else first for i in ins], shape[2] * shape[3]
        return [first, _like(first, dev, stream)], shape[2] * shape[3]
    outs = [None if i is None else _like(i, dev, stream) if o is None else o
            for o, i in zip(outs, ins)]
    for n, o, i in zip(names, outs, ins):
        if o is not None:
            _heads(n, o, i)
    return outs, _tok_stride(*_given(*outs))


def qk_rotary(rotary: Rotary, q, k, positions, q_norm=None, k_norm=None, eps: float = 1e-6, q_out=None, k_out=None,
              stream=None):
    """RMS norm (where a weight is given) and rotation of queries and keys.
    q, k: [B, N, H, D] bf16 views with one token stride, either may be None;
    positions: [N, axes] or [B, N, axes], int32 or float32; q_norm, k_norm:
    [D] bf16.  q_out may be q and k_out k (in place).  Returns (q_out, k_out)."""
    given = _pair(("q", "k"), q, k, rotary.head_dim)
    B, N, H, D = given[0].shape
    dev = given[0].device
    pf, pb = _positions(rotary, given[0], positions)
    _norm_weight("q_norm", q_norm, D)
    _norm_weight("k_norm", k_norm, D)
    ts = _tok_stride(*given)
    (qo, ko), os_ = _outputs((q_out, k_out), (q, k), ("q_out", "k_out"), dev, stream)
    _same_device(dev, positions=positions, q_norm=q_norm, k_norm=k_norm)
    _call(lib().rc_qk_rotary, dev, stream, ctypes.byref(rotary.c), B, N, H, _ptr(q), _ptr(k), ts, positions.data_ptr(),
          pf, pb, _ptr(q_norm), _ptr(k_norm), eps, _ptr(qo), _ptr(ko), os_)
    return qo, ko


def qk_rotary_backward(rotary: Rotary, dq, dk, positions, q=None, k=None, q_norm=None, k_norm=None, eps: float = 1e-6,
                       dq_out=None, dk_out=None, workspace=None, stream=None):
    """Gradient of qk_rotary: dq, dk are the gradients of its outputs; q, k its
    inputs, needed where there is a norm.  dq_out may be dq and dk_out dk.
    Returns (dq_out, dk_out, dq_norm, dk_norm); the norms' gradients are [D] fp32."""
    torch = _torch()
    given = _pair(("dq", "dk"), dq, dk, rotary.head_dim)
    B, N, H, D = given[0].shape
    dev = given[0].device
    pf, pb = _positions(rotary, given[0], positions)
    _norm_weight("q_norm", q_norm, D)
    _norm_weight("k_norm", k_norm, D)
    inputs = []
    for name, w, t, g in (("q", q_norm, q, dq), ("k", k_norm, k, dk)):
        if w is not None:
            if t is None or g is None:
                raise ValueError(f"{name}_norm needs {name} and d{name}")
            _heads(name, t, g)
            inputs.append(t)
    ts = _tok_stride(*inputs) if inputs else 0
    gs = _tok_stride(*given)
    (qo, ko), os_ = _outputs((dq_out, dk_out), (dq, dk), ("dq_out", "dk_out"), dev, stream)
    dw = [_empty((D,), torch.float32, dev, stream) if w is not None else None for w in (q_norm, k_norm)]
    need = int(lib().rc_rotary_backward_workspace_bytes(ctypes.byref(rotary.c), B, N)) if inputs else 0
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _empty(need, torch.uint8, dev, stream, returned=False)
    _same_device(dev, positions=positions, q_norm=q_norm, k_norm=k_norm, workspace=workspace if need else None)
    _call(lib().rc_qk_rotary_backward, dev, stream, ctypes.byref(rotary.c), B, N, H, _ptr(dq), _ptr(dk), gs,
          positions.data_ptr(), pf, pb, _ptr(q if q_norm is not None else None), _ptr(k if k_norm is not None else None),
          ts, _ptr(q_norm), _ptr(k_norm), eps, _ptr(qo), _ptr(ko), os_, _ptr(dw[0]), _ptr(dw[1]),
          _ptr(workspace) if need else None, need)
    return qo, ko, dw[0], dw[1]


# ---------------------------------------------------------------- gated norm between blocks
NORMS = {"layer": 0, "rms": 1}
_I32S = ctypes.c_int32 * RC_MAX_SEGMENTS
NormGrads = collections.namedtuple("NormGrads", "h x gate scale shift weight post_weight")


def _row_stride(name, t, like=None, ld=0):
    """Row stride of a bf16 [B, N, C] GPU tensor with C contiguous and batch stride N row strides.
    The first test covers a tensor laid out as `like`, whose row stride is ld."""
    if like is not None:
        if (t.stride() == like.stride() and t.shape == like.shape and t.dtype is _torch().bfloat16
                and t.device == like.device):
            return ld
    if t.dim() != 3 or t.dtype is not _torch().bfloat16 or not t.is_cuda:
        raise ValueError(f"{name} must be a bf16 [B, N, C] GPU tensor, got {str(t.dtype)} {tuple(t.shape)} on {t.device}")
    if like is not None and (t.shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must have shape {tuple(like.shape)} on {like.device}, got {tuple(t.shape)} on {t.device}")
    B, N, C = t.shape
    sb, sn, sc = t.stride()
    if C > 1 and sc != 1:
        raise ValueError(f"{name} must have unit channel stride")
    if N <= 1:
        return sb if N == 1 and B > 1 else C
    if B > 1 and sb != N * sn:
        raise ValueError(f"{name} must have batch stride N * row stride")
    return sn


def _norm_desc(h, spans, norm, post, eps, residual_scale, mods, weight, post_weight):
    """rc_norm of a call: shapes, spans and the strides that gate, scale and
    shift share (a vector laid out as the first one needs no other check)."""
    bf16, dev = _torch().bfloat16, h.device
    B, N, C = h.shape
    kind = NORMS.get(norm)
    if kind is None:
        raise ValueError(f"norm must be one of {sorted(NORMS)}, got {norm!r}")
    if spans is None:
        rows, groups, G = (N,), (0,), 1
    else:
        if len(spans) > RC_MAX_SEGMENTS:
            raise ValueError(f"at most {RC_MAX_SEGMENTS} spans")
        rows, groups = zip(*spans) if spans else ((), ())
        G = max(groups, default=0) + 1
    first = strides = None
    mod_batch = mod_group = 0
    for name, t in mods:
        if t is None:
            continue
        if first is not None and (t.stride() == first.stride() and t.shape == first.shape and t.dtype is bf16
                                  and t.device == dev):
            continue
        if t.dim() != 3 or t.dtype is not bf16 or t.shape[0] != B or t.shape[2] != C or t.device != dev:
            raise ValueError(f"{name} must be a bf16 [{B}, groups, {C}] tensor on {h.device}, got {str(t.dtype)} "
                             f"{tuple(t.shape)} on {t.device}")
        sb, sg, sc = t.stride()
        n = t.shape[1]
        if C > 1 and sc != 1:
            raise ValueError(f"{name} must have unit channel stride")
        mine = (n, sb if B > 1 else 0, sg if n > 1 else 0)
        if strides is not None and mine != strides:
            raise ValueError("gate, scale and shift must share groups and strides (chunks of one tensor do)")
        first, strides = t, mine
    if strides is not None:
        G, mod_batch, mod_group = strides
    if weight is not None or post_weight is not None:
        for name, w in (("weight", weight), ("post_weight", post_weight)):
            _norm_weight(name, w, C)
        _same_device(h.device, weight=weight, post_weight=post_weight)
    return rc_norm(B, C, G, kind, post, N, eps, residual_scale, mod_batch, mod_group, len(rows),
                   _I32S(*rows), _I32S(*groups)), G


def gated_norm(h, x=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, norm: str = "layer",
               post_norm: bool = False, spans=None, residual_scale: float = 1.0, eps: float = 1e-6, h_out=None, y=None,
               want_y: bool = True, stream=None):
    """h' = h + residual_scale * gate * u, with u = x or (post_norm, implied by
    post_weight) the RMS norm of x, and y = norm(h') * weight * (1 + scale) + shift.

    h, x: [B, N, C] bf16 rows; gate, scale, shift: [B, groups, C] (chunks of
    one modulation tensor work); weight, post_weight: [C]; spans: (rows,
    group) pairs over N, e.g. Layout.modulation_spans (None: one group).
    Returns (h', y); h_out may be h.  Without x, h' is h itself; want_y=False
    computes the residual alone."""
    ldh = _row_stride("h", h)
    dev, C = h.device, h.shape[2]
    post = post_norm or post_weight is not None
    d, _ = _norm_desc(h, spans, norm, post, eps, residual_scale, (("gate", gate), ("scale", scale), ("shift", shift)),
                      weight, post_weight)
    ldx = ldo = ldy = 0
    if x is not None:
        ldx = _row_stride("x", x, h, ldh)
        if h_out is None:
            h_out, ldo = _like(h, dev, stream), C
        else:
            ldo = _row_stride("h_out", h_out, h, ldh)
    elif h_out is not None:
        raise ValueError("h_out is written only with x")
    if not want_y:
        if y is not None:
            raise ValueError("y is written only with want_y")
    elif y is None:
        y, ldy = _like(h, dev, stream), C
    else:
        ldy = _row_stride("y", y, h, ldh)
    _call(lib().rc_gated_norm, dev, stream, ctypes.byref(d), h.data_ptr(), ldh, _ptr(x), ldx, _ptr(gate), _ptr(scale),
          _ptr(shift), _ptr(weight), _ptr(post_weight), _ptr(h_out), ldo, _ptr(y), ldy)
    return (h if x is None else h_out), y


def gated_norm_backward(dy, h, x=None, dh=None, gate=None, scale=None, shift=None, weight=None, post_weight=None,
                        norm: str = "layer", post_norm: bool = False, spans=None, residual_scale: float = 1.0,
                        eps: float = 1e-6, dh_out=None, dx=None, workspace=None, stream=None):
    """Gradient of gated_norm at its output rows h (= h').  dy: the gradient of
    y (None: none); dh: the gradient of h' from elsewhere (None: none); the
    other arguments as the forward's.  dh_out may be dh or dy, dx may be x.
    Returns NormGrads(h, x, gate, scale, shift, weight, post_weight): the rows'
    in bf16, the shared ones in fp32 ([B, groups, C] and [C]), None where the
    forward had none."""
    torch = _torch()
    ldh = _row_stride("h", h)
    dev = h.device
    post = post_norm or post_weight is not None
    d, G = _norm_desc(h, spans, norm, post, eps, residual_scale, (("gate", gate), ("scale", scale), ("shift", shift)),
                      weight, post_weight)
    B, _, C = h.shape
    lddy = _row_stride("dy", dy, h, ldh) if dy is not None else 0
    lddh = _row_stride("dh", dh, h, ldh) if dh is not None else 0
    ldx = lddx = 0
    if dh_out is None:
        dh_out, ldo = _like(h, dev, stream), C
    else:
        ldo = _row_stride("dh_out", dh_out, h, ldh)
    if x is not None:
        ldx = _row_stride("x", x, h, ldh)
        if dx is None:
            dx, lddx = _like(h, dev, stream), C
        else:
            lddx = _row_stride("dx", dx, h, ldh)
    elif dx is not None:
        raise ValueError("dx is written only with x")
    shared = None
    vectors = [None, None, None]
    for i, t in enumerate((gate, scale, shift)):
        if t is not None:
            shared = _empty((B, G, C), torch.float32, dev, stream) if shared is None else _like(shared, dev, stream)
            vectors[i] = shared
    dgate, dscale, dshift = vectors
    dweight, dpost = (None if w is None else _empty((C,), torch.float32, dev, stream) for w in (weight, post_weight))
    need = int(lib().rc_gated_norm_backward_workspace_bytes(ctypes.byref(d)))
    if workspace is not None:
        _same_device(dev, workspace=workspace if need else None)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _empty(need, torch.uint8, dev, stream, returned=False)
    _call(lib().rc_gated_norm_backward, dev, stream, ctypes.byref(d), _ptr(dy), lddy, _ptr(dh), lddh, h.data_ptr(), ldh,
          _ptr(x), ldx, _ptr(gate), _ptr(scale), _ptr(weight), _ptr(post_weight), dh_out.data_ptr(), ldo, _ptr(dx), lddx,
          _ptr(dgate), _ptr(dscale), _ptr(dshift), _ptr(dweight), _ptr(dpost), _ptr(workspace) if need else None, need)
    return NormGrads(dh_out, dx, dgate, dscale, dshift, dweight, dpost)


# ---------------------------------------------------------------- FP8 reference cache
def fp8_cache_shapes(layout: Layout, B: int, H: int, D: int):
    """Shapes of the FP8 cache: K8 and V8 [B, H, N_cached, D] (uint8 e4m3fn
    codes, the rows of the bf16 cache) and the scales [B, H, 2] (fp32)."""
    n = layout.rows(ROWS_CACHED)
    return (B, H, n, D), (B, H, n, D), (B, H, 2)


def ref_kv_prefill_fp8(layout: Layout, q, k, v, o=None, lse=None, k_cache8=None, v_cache8=None, kv_scale=None,
                       scale: Optional[float] = None, want_lse: bool = False, stream=None):
    """Static-subgraph prefill writing the FP8 cache.  Returns
    (o, lse or None, k_cache8, v_cache8, kv_scale)."""
    torch = _torch()
    _rows_of(layout, q, ROWS_STATIC, "ref_kv_prefill_fp8")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    ks, vs, ss = fp8_cache_shapes(layout, B, H, D)
    if o is None:
        o = _empty((B, N, H, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _empty((B, H, N), torch.float32, dev, stream)
    if k_cache8 is None:
        k_cache8 = _empty(ks, torch.uint8, dev, stream)
    if v_cache8 is None:
        v_cache8 = _empty(vs, torch.uint8, dev, stream)
    if kv_scale is None:
        kv_scale = _empty(ss, torch.float32, dev, stream)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(k_cache8, ks, "torch.uint8", "k_cache8")
    _expect(v_cache8, vs, "torch.uint8", "v_cache8")
    _expect(kv_scale, ss, "torch.float32", "kv_scale")
    _same_device(dev, o=o, lse=lse, k_cache8=k_cache8, v_cache8=v_cache8, kv_scale=kv_scale)
    _call(lib().rc_ref_kv_prefill_fp8, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(), k.data_ptr(),
          v.data_ptr(), ts, o.data_ptr(), _ptr(lse), k_cache8.data_ptr(), v_cache8.data_ptr(), kv_scale.data_ptr())
    return o, lse, k_cache8, v_cache8, kv_scale


def step_masked_attention_fp8(layout: Layout, q, k, v, k_cache8, v_cache8, kv_scale, o=None, lse=None,
                              splits: int = 0, workspace=None, scale: Optional[float] = None, want_lse: bool = False,
                              stream=None):
    """Per-step attention reading the FP8 cache (fresh LT/X K/V stay bf16).
    Returns (o, lse or None)."""
    torch = _torch()
    _rows_of(layout, q, ROWS_LIVE, "step_masked_attention_fp8")
    dev = _inputs(q, k, v)
    B, N, H, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ts = _tok_stride(q, k, v)
    ks, vs, ss = fp8_cache_shapes(layout, B, H, D)
    if o is None:
        o = _empty((B, N, H, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _empty((B, H, N), torch.float32, dev, stream)
    _expect(o, (B, N, H, D), "torch.bfloat16", "o")
    _expect(lse, (B, H, N), "torch.float32", "lse")
    _expect(k_cache8, ks, "torch.uint8", "k_cache8")
    _expect(v_cache8, vs, "torch.uint8", "v_cache8")
    _expect(kv_scale, ss, "torch.float32", "kv_scale")
    need = layout.workspace_bytes(B, H, D, splits) if splits != SPLITS_BALANCED else 0
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _empty(need, torch.uint8, dev, stream, returned=False)
    _same_device(dev, o=o, lse=lse, k_cache8=k_cache8, v_cache8=v_cache8, kv_scale=kv_scale,
                 workspace=workspace if need else None)
    _call(lib().rc_step_masked_attention_fp8, dev, stream, ctypes.byref(layout.c), B, H, D, scale, q.data_ptr(),
          k.data_ptr(), v.data_ptr(), ts, k_cache8.data_ptr(), v_cache8.data_ptr(), kv_scale.data_ptr(), o.data_ptr(),
          _ptr(lse), splits, _ptr(workspace) if need else None, need)
    return o, lse
