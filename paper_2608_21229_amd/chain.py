"""Chained synthetic DiT layers on the library's kernels.

Each layer projects its input hidden state to Q, K and V (Sec. 3.1, Eq. 2:
a layer's K and V are projections of that layer's input), runs the masked
attention, and adds the output projection to the residual:

    qkv = h W_qkv^T            rc_linear; W_qkv rows are the Q heads, then the
                               K heads, then the V heads (D each)
    O   = attention(Q, K, V)   Q/K/V are strided views of qkv (token stride 3 H D)
    h'  = h + O W_o^T          rc_linear with the residual

Optionally (``rotary``, ``q_norms``/``k_norms``, ``modulated``) a layer also has what
such layers have around the attention, by the library's kernels:

    y   = norm(h) (1 + scale) + shift           gated_norm; modulation by segment: live
                                                rows take group 0, static rows group 1
    Q,K = rotation(norm(Q, K)) by position      qk_rotary, in place in the fused buffer
    h'  = h + gate * (O W_o^T)                  gated_norm, fused with the next layer's norm

Four ways through the stack:
    prefill  the static rows (ST and R) through every layer; each layer's
             attention stores that layer's reference K/V cache
    step     the live rows (LT and X) through every layer over those caches
    full     every row through every layer: the recompute baseline, in which
             every token is re-projected and attended at each step
    full_backward  the gradient of the recompute, for training under the mask

With ``cache="fp8"`` each layer's reference cache is stored as e4m3 codes
with per-(batch, head) scales (``ref_kv_prefill_fp8`` /
``step_masked_attention_fp8``); the computation stays bf16.

Every multiply-add runs in librefcache.  Work buffers come from torch's
allocator; ``collect`` (a list) receives a copy of the hidden state after each
layer.  ``full_backward`` also copies with torch: the weights transposed, and for
the weights' gradients both activations of a product transposed and padded.  With ``stream`` given, everything that a call
allocates, copies and launches is that stream's.
"""
from __future__ import annotations

import collections
import contextlib
import math
from typing import List, Optional, Sequence, Tuple

from . import binding as rcb


class Chain:
    """A stack of synthetic layers with fixed weights and block mask.

    w_qkv[l]: [3 H D, H D] bf16, w_o[l]: [H D, H D] bf16, on one GPU.
    rotary: a Rotary, with positions [N, axes] of all tokens in sequence order,
    copied here (later writes to the caller's tensor change nothing; keep the
    chain as long as a graph that captured its calls is replayed);
    q_norms, k_norms: a [D] weight per layer; modulated: every call takes
    ``modulation`` [B, groups, layers, 3, H D] (shift, scale, gate per layer):
    one group for prefill and step, two (live, static) for full."""

    def __init__(self, layout: rcb.Layout, w_qkv: Sequence, w_o: Sequence, H: int, D: int,
                 scale: Optional[float] = None, cache: str = "bf16", rotary: Optional[rcb.Rotary] = None,
                 positions=None, q_norms: Optional[Sequence] = None, k_norms: Optional[Sequence] = None,
                 modulated: bool = False, norm: str = "layer", eps: float = 1e-6):
        if len(w_qkv) != len(w_o) or not w_qkv:
            raise ValueError("need one W_qkv and one W_o per layer")
        if cache not in ("bf16", "fp8"):
            raise ValueError(f"cache must be 'bf16' or 'fp8', got {cache!r}")
        self.cache = cache
        C = H * D
        for l, (wq, wo) in enumerate(zip(w_qkv, w_o)):
            if tuple(wq.shape) != (3 * C, C) or tuple(wo.shape) != (C, C):
                raise ValueError(f"layer {l}: W_qkv must be [{3 * C}, {C}] and W_o [{C}, {C}], "
                                 f"got {tuple(wq.shape)} and {tuple(wo.shape)}")
        self.layout, self.w_qkv, self.w_o = layout, list(w_qkv), list(w_o)
        self.H, self.D, self.C = H, D, C
        self.scale = 1.0 / math.sqrt(D) if scale is None else scale
        if (rotary is None) != (positions is None):
            raise ValueError("rotary and positions go together")
        if (q_norms is None) != (k_norms is None):
            raise ValueError("q_norms and k_norms go together")
        if q_norms is not None and (rotary is None or not len(q_norms) == len(k_norms) == len(self.w_qkv)):
            raise ValueError("q_norms and k_norms need rotary and one weight per layer")
        if positions is not None and (positions.dim() != 2 or positions.shape[0] != layout.rows(rcb.ROWS_ALL)):
            raise ValueError(f"positions must be [{layout.rows(rcb.ROWS_ALL)}, axes], got {tuple(positions.shape)}")
        self.rotary, self.q_norms, self.k_norms = rotary, q_norms, k_norms
        self.modulated, self.norm, self.eps = modulated, norm, eps
        self._positions = {}
        if positions is not None:
            # a copy, as the gathered rows below are: the cached path and the recompute stay of one mind
            positions = positions.clone(memory_format=rcb._torch().contiguous_format)
            self._positions[rcb.ROWS_ALL] = positions
            for which in (rcb.ROWS_STATIC, rcb.ROWS_LIVE):
                self._positions[which] = self._rows_of(positions, which)
            # gathered on the stream that is current here, read on every call's
            if positions.is_cuda:
                rcb._torch().cuda.current_stream(positions.device).synchronize()

    def _rows_of(self, t, which: int):
        """The rows of a class out of a tensor over all tokens."""
        parts, at = [], 0
        for kind, n in self.layout.segments:
            if (kind in (rcb.SEG_TEXT, rcb.SEG_TARGET)) == (which == rcb.ROWS_LIVE):
                parts.append(t[at:at + n])
            at += n
        return rcb._torch().cat(parts).contiguous() if parts else t[:0]

    def _mod(self, modulation, rows_kind: int, B: int):
        """Checked modulation of a call, and the spans of its rows."""
        if not self.modulated:
            if modulation is not None:
                raise ValueError("modulation needs a Chain with modulated=True")
            return None
        groups = 2 if rows_kind == rcb.ROWS_ALL else 1
        want = (B, groups, self.layers, 3, self.C)
        if modulation is None or tuple(modulation.shape) != want:
            raise ValueError(f"modulation must be {want}, got {None if modulation is None else tuple(modulation.shape)}")
        return modulation

    def _spans(self, rows_kind: int):
        return self.layout.modulation_spans(rows_kind, live=0, static=1 if rows_kind == rcb.ROWS_ALL else 0)

    def _norms(self, l: int):
        return (None, None) if self.q_norms is None else (self.q_norms[l], self.k_norms[l])

    @property
    def layers(self) -> int:
        return len(self.w_qkv)

    @contextlib.contextmanager
    def _scope(self, stream, dev):
        """Makes the caller's stream the current one; yields a function that
        marks tensors to be returned as used on the stream that was current."""
        if stream is None:
            yield lambda *ts: None
            return
        caller = rcb._torch().cuda.current_stream(dev)
        with rcb._on(stream, dev):
            yield lambda *ts: [t.record_stream(caller) for t in ts]

    def _read_positions(self, rows_kind: int, dev):
        """Marks a call's positions as read on the stream that is current (with
        stream= the call's): they belong to the constructor's, nobody but the
        chain holds them, and it may be dropped before they have been read."""
        t = self._positions.get(rows_kind)
        if t is not None and t.device == dev:  # elsewhere: the rotation refuses them
            t.record_stream(rcb._torch().cuda.current_stream(dev))

    def _check_rows(self, h, rows_kind: int):
        if h.dim() != 3 or h.shape[2] != self.C:
            raise ValueError(f"hidden state must be [B, N, {self.C}], got {tuple(h.shape)}")
        B, N, _ = h.shape
        want = self.layout.rows(rows_kind)
        if N != want:
            raise ValueError(f"hidden state has {N} rows, the layout {want}")
        return B, N

    def _buffers(self, h, rows_kind: int):
        torch = rcb._torch()
        B, N = self._check_rows(h, rows_kind)
        qkv = torch.empty((B * N, 3 * self.C), dtype=torch.bfloat16, device=h.device)
        o = torch.empty((B, N, self.H, self.D), dtype=torch.bfloat16, device=h.device)
        work = torch.empty((B * N, self.C), dtype=torch.bfloat16, device=h.device)
        return B, N, qkv, o, work

    def _qkv_views(self, qkv, B, N):
        t = qkv.view(B, N, 3, self.H, self.D)
        return t[:, :, 0], t[:, :, 1], t[:, :, 2]

    def _run(self, h, rows_kind, attend, collect: Optional[List], last_out: bool = True, stream=None, modulation=None):
        with self._scope(stream, h.device) as returned:
            n = len(collect) if collect is not None else 0
            out = self._layers(h, rows_kind, attend, collect, last_out, stream, modulation)
            returned(out, *(collect[n:] if collect is not None else ()))
            return out

    def _rotate(self, l, q, k, rows_kind, stream, q_out=None, k_out=None):
        if self.rotary is None:
            return q, k
        q_norm, k_norm = self._norms(l)
        return rcb.qk_rotary(self.rotary, q, k, self._positions[rows_kind], q_norm=q_norm, k_norm=k_norm, eps=self.eps,
                             q_out=q if q_out is None else q_out, k_out=k if k_out is None else k_out, stream=stream)

    def _layers(self, h, rows_kind, attend, collect, last_out, stream, modulation):
        B, N, qkv, o, work = self._buffers(h, rows_kind)
        self._read_positions(rows_kind, h.device)
        mod = self._mod(modulation, rows_kind, B)
        if mod is not None:
            return self._modulated_layers(h, rows_kind, attend, collect, last_out, stream, mod, B, N, qkv, o, work)
        src = h.reshape(B * N, self.C)
        for l in range(self.layers):
            rcb.linear(src, self.w_qkv[l], out=qkv, stream=stream)
            q, k, v = self._qkv_views(qkv, B, N)
            self._rotate(l, q, k, rows_kind, stream)
            attend(l, q, k, v, o)
            if l + 1 < self.layers or last_out or collect is not None:
                rcb.linear(o.view(B * N, self.C), self.w_o[l], residual=src, out=work, stream=stream)
                src = work
                if collect is not None:
                    collect.append(work.view(B, N, self.C).clone())
        return src.view(B, N, self.C)

    def _modulated_layers(self, h, rows_kind, attend, collect, last_out, stream, mod, B, N, qkv, o, work):
        spans = self._spans(rows_kind)
        y = rcb._torch().empty_like(work).view(B, N, self.C)
        branch = work.view(B, N, self.C)
        h = h.reshape(B, N, self.C)
        rcb.gated_norm(h, scale=mod[:, :, 0, 1], shift=mod[:, :, 0, 0], norm=self.norm, eps=self.eps, spans=spans, y=y,
                       stream=stream)
        out = None  # the hidden state from the first layer's residual on
        for l in range(self.layers):
            rcb.linear(y.view(B * N, self.C), self.w_qkv[l], out=qkv, stream=stream)
            q, k, v = self._qkv_views(qkv, B, N)
            self._rotate(l, q, k, rows_kind, stream)
            attend(l, q, k, v, o)
            last = l + 1 == self.layers
            if last and not last_out and collect is None:
                break
            rcb.linear(o.view(B * N, self.C), self.w_o[l], out=work, stream=stream)
            nxt = {} if last else dict(scale=mod[:, :, l + 1, 1], shift=mod[:, :, l + 1, 0], y=y)
            h, _ = rcb.gated_norm(h, branch, gate=mod[:, :, l, 2], norm=self.norm, eps=self.eps, spans=spans, h_out=out,
                                  want_y=not last, stream=stream, **nxt)
            out = h
            if collect is not None:
                collect.append(h.clone())
        return h

    def new_caches(self, B: int, device) -> List[Tuple]:
        """Per layer (K_cache, V_cache) bf16, or (K8, V8, scales) for the FP8 cache."""
        torch = rcb._torch()
        if self.cache == "fp8":
            ks, vs, ss = rcb.fp8_cache_shapes(self.layout, B, self.H, self.D)
            return [(torch.empty(ks, dtype=torch.uint8, device=device),
                     torch.empty(vs, dtype=torch.uint8, device=device),
                     torch.empty(ss, dtype=torch.float32, device=device)) for _ in range(self.layers)]
        nc = self.layout.rows(rcb.ROWS_CACHED)
        shape = (B, self.H, nc, self.D)
        return [(torch.empty(shape, dtype=torch.bfloat16, device=device),
                 torch.empty(shape, dtype=torch.bfloat16, device=device)) for _ in range(self.layers)]

    def prefill(self, h_static, caches=None, collect: Optional[List] = None, stream=None, modulation=None):
        """h_static [B, N_static, H D]: the ST and R rows in sequence order.
        Fills and returns one cache entry per layer (see ``new_caches``).  The static
        rows' output projection of the last layer is skipped (nobody reads
        it) unless ``collect`` asks for the hidden states."""
        if caches is None:
            with self._scope(stream, h_static.device) as returned:
                caches = self.new_caches(h_static.shape[0], h_static.device)
                returned(*(t for entry in caches for t in entry))
        if len(caches) != self.layers:
            raise ValueError(f"need {self.layers} cache entries, got {len(caches)}")

        def attend(l, q, k, v, o):
            if self.cache == "fp8":
                rcb.ref_kv_prefill_fp8(self.layout, q, k, v, o=o, k_cache8=caches[l][0], v_cache8=caches[l][1],
                                       kv_scale=caches[l][2], scale=self.scale, stream=stream)
            else:
                rcb.ref_kv_prefill(self.layout, q, k, v, o=o, k_cache=caches[l][0], v_cache=caches[l][1],
                                   scale=self.scale, stream=stream)

        self._run(h_static, rcb.ROWS_STATIC, attend, collect, last_out=False, stream=stream, modulation=modulation)
        return caches

    def step(self, h_live, caches, splits: int = 0, collect: Optional[List] = None, stream=None, modulation=None):
        """h_live [B, N_live, H D]: the LT and X rows of one denoising step.
        Returns the live rows' hidden state after the last layer."""
        if len(caches) != self.layers:
            raise ValueError(f"need {self.layers} cache entries, got {len(caches)}")
        B = h_live.shape[0]
        need = self.layout.workspace_bytes(B, self.H, self.D, splits)
        ws = rcb._empty(need, rcb._torch().uint8, h_live.device, stream, returned=False) if need else None

        def attend(l, q, k, v, o):
            if self.cache == "fp8":
                rcb.step_masked_attention_fp8(self.layout, q, k, v, *caches[l], o=o, splits=splits, workspace=ws,
                                              scale=self.scale, stream=stream)
            else:
                rcb.step_masked_attention(self.layout, q, k, v, caches[l][0], caches[l][1], o=o, splits=splits,
                                          workspace=ws, scale=self.scale, stream=stream)

        return self._run(h_live, rcb.ROWS_LIVE, attend, collect, stream=stream, modulation=modulation)

    def full(self, h, collect: Optional[List] = None, stream=None, last_round_split: bool = True, modulation=None):
        """h [B, N, H D]: every row in sequence order.  Returns the hidden state
        after the last layer.  last_round_split=False computes every query tile
        whole (bit-comparable with the cached path)."""
        def attend(l, q, k, v, o):
            rcb.full_attention(self.layout, q, k, v, o=o, scale=self.scale, last_round_split=last_round_split,
                               stream=stream)

        return self._run(h, rcb.ROWS_ALL, attend, collect, stream=stream, modulation=modulation)

    def full_backward(self, h, dh, modulation=None, stream=None) -> "ChainGrads":
        """Gradient of ``full``: dh [B, N, H D] is the gradient of its result.
        Runs the layers forward, keeping their activations, and back.  Returns
        ChainGrads(h, w_qkv, w_o, q_norms, k_norms, modulation): the hidden
        state's and the weights' in bf16, the norms' and the modulation's in
        fp32 (None where the chain has none)."""
        with self._scope(stream, h.device) as returned:
            grads = self._full_backward(h, dh, modulation, stream)
            for g in grads:
                if g is not None:
                    returned(*(g if isinstance(g, list) else [g]))
            return grads

    def _full_backward(self, h, dh, modulation, stream):
        torch = rcb._torch()
        B, N = self._check_rows(h, rcb.ROWS_ALL)
        C, M = self.C, B * N
        if tuple(dh.shape) != tuple(h.shape):
            raise ValueError(f"dh must be {tuple(h.shape)}, got {tuple(dh.shape)}")
        mod = self._mod(modulation, rcb.ROWS_ALL, B)
        self._read_positions(rcb.ROWS_ALL, h.device)
        spans = self._spans(rcb.ROWS_ALL)
        norm = dict(norm=self.norm, eps=self.eps, spans=spans, stream=stream)
        kept, h = [], h.contiguous()
        first = h
        y = h if mod is None else rcb.gated_norm(h, scale=mod[:, :, 0, 1], shift=mod[:, :, 0, 0], **norm)[1]
        for l in range(self.layers):
            qkv = rcb.linear(y.view(M, C), self.w_qkv[l], stream=stream)
            q, k, v = self._qkv_views(qkv, B, N)
            turned = qkv
            if self.q_norms is not None:  # the norm's gradient reads its inputs
                turned = qkv.clone()
            elif self.rotary is not None:
                qkv = None
            qt, kt, vt = self._qkv_views(turned, B, N)
            self._rotate(l, q, k, rcb.ROWS_ALL, stream, qt, kt)
            o, lse = rcb.full_attention(self.layout, qt, kt, vt, scale=self.scale, want_lse=True, stream=stream)
            last = l + 1 == self.layers
            if mod is None:
                branch, at = None, h
                h = y_next = rcb.linear(o.view(M, C), self.w_o[l], residual=h.view(M, C), stream=stream).view(B, N, C)
            else:
                branch = rcb.linear(o.view(M, C), self.w_o[l], stream=stream).view(B, N, C)
                nxt = {} if last else dict(scale=mod[:, :, l + 1, 1], shift=mod[:, :, l + 1, 0])
                at, y_next = rcb.gated_norm(h, branch, gate=mod[:, :, l, 2], want_y=not last, **nxt, **norm)
                h = at
            kept.append((y, qkv, turned, o, lse, branch, at))
            y = y_next

        d_qkv, d_o = [None] * self.layers, [None] * self.layers
        dq_norms = dk_norms = None
        if self.q_norms is not None:
            dq_norms, dk_norms = [None] * self.layers, [None] * self.layers
        dmod = None if mod is None else torch.zeros(mod.shape, dtype=torch.float32, device=mod.device)
        dh, dy = dh.contiguous(), None
        for l in reversed(range(self.layers)):
            y, qkv, turned, o, lse, branch, at = kept.pop()
            last = l + 1 == self.layers
            if mod is None:
                da = dh
            else:
                nxt = {} if last else dict(scale=mod[:, :, l + 1, 1], shift=mod[:, :, l + 1, 0])
                g = rcb.gated_norm_backward(dy, at, branch, dh=dh, gate=mod[:, :, l, 2], **nxt, **norm)
                dh, da, dmod[:, :, l, 2] = g.h, g.x, g.gate
                if not last:
                    dmod[:, :, l + 1, 0], dmod[:, :, l + 1, 1] = g.shift, g.scale
            d_o[l] = _weight_grad(da.view(M, C), o.view(M, C), stream)
            do = rcb.linear(da.view(M, C), self.w_o[l].t().contiguous(), stream=stream).view(B, N, self.H, self.D)
            q, k, v = self._qkv_views(turned, B, N)
            dqkv = torch.empty_like(turned)
            dq, dk, dv = self._qkv_views(dqkv, B, N)
            rcb.full_attention_backward(self.layout, q, k, v, o, lse, do, dq, dk, dv, scale=self.scale, stream=stream)
            if self.rotary is not None:
                q_norm, k_norm = self._norms(l)
                q0, k0 = (None, None) if q_norm is None else self._qkv_views(qkv, B, N)[:2]
                _, _, gq, gk = rcb.qk_rotary_backward(self.rotary, dq, dk, self._positions[rcb.ROWS_ALL], q=q0, k=k0,
                                                      q_norm=q_norm, k_norm=k_norm, eps=self.eps, dq_out=dq, dk_out=dk,
                                                      stream=stream)
                if q_norm is not None:
                    dq_norms[l], dk_norms[l] = gq, gk
            d_qkv[l] = _weight_grad(dqkv, y.reshape(M, C), stream)
            w_t = self.w_qkv[l].t().contiguous()
            if mod is None:
                dh = rcb.linear(dqkv, w_t, residual=dh.view(M, C), stream=stream).view(B, N, C)
            else:
                dy = rcb.linear(dqkv, w_t, stream=stream).view(B, N, C)
        if mod is not None:
            g = rcb.gated_norm_backward(dy, first, dh=dh, scale=mod[:, :, 0, 1], shift=mod[:, :, 0, 0], **norm)
            dh, dmod[:, :, 0, 0], dmod[:, :, 0, 1] = g.h, g.shift, g.scale
        return ChainGrads(dh, d_qkv, d_o, dq_norms, dk_norms, dmod)


ChainGrads = collections.namedtuple("ChainGrads", "h w_qkv w_o q_norms k_norms modulation")


def _weight_grad(dy, x, stream):
    """dy^T x [n, k] of dy [M, n] and x [M, k] by the projection kernel, whose
    inner length is a multiple of 64: rows of zeros fill M up."""
    torch = rcb._torch()
    M = dy.shape[0]
    pad = -M % 64
    t = lambda a: torch.nn.functional.pad(a.t(), (0, pad)).contiguous()  # noqa: E731
    return rcb.linear(t(dy), t(x), stream=stream)
