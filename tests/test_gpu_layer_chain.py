"""The layer operators together, as a chain of layers uses them: modulated
norm, projection, norm and rotation of queries and keys, masked attention,
output projection, gated residual -- cached and recomputed, and the gradient.

Exactness: every part but the attention works row by row in a fixed order, so
the cached path's live rows equal the recompute's bit for bit where the plain
chain's do (segments on the 64-key grid, whole tiles).

Gradient: against the same chain in 64 bits, differentiated by torch.  The
library's chain stores some 9 tensors a layer forward and 9 back in bf16, each
off by 2^-8 / sqrt(3) of its size in the root mean square and independent of
the others: sqrt(18 layers) 2^-8 / sqrt(3) = 1.4e-2 for two layers, and what
passes through the softmax and the norms is carried with a gain of the order
of one; 3e-2 of a gradient's L2 norm is allowed."""
import pytest
import torch

import paper_2608_21229_amd as rc
from synthgen import bf16_normal, derive_seed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
REL = 3e-2


def draw(shape, seed, i, std=1.0):
    return bf16_normal(tuple(shape), derive_seed(seed, 0, 0, i), std).to(DEV)


def make(segs, mask, B, H, D, layers, seed, modulated=True, rotary=True, norms=True, kind="layer", interleaved=True):
    L = rc.Layout(segs, mask)
    C, N = H * D, sum(n for _, n in segs)
    w_qkv = [draw((3 * C, C), seed, 10 + l, C ** -0.5) for l in range(layers)]
    w_o = [draw((C, C), seed, 20 + l, C ** -0.5) for l in range(layers)]
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(-32, 32, (N, 3), generator=g, dtype=torch.int32).to(DEV) if rotary else None
    R = rc.Rotary(D, (16, 24, 24) if D == 64 else (16, 56, 56), interleaved=interleaved) if rotary else None
    qn = [1 + draw((D,), seed, 30 + l, 0.2) for l in range(layers)] if rotary and norms else None
    kn = [1 + draw((D,), seed, 40 + l, 0.2) for l in range(layers)] if rotary and norms else None
    chain = rc.Chain(L, w_qkv, w_o, H, D, rotary=R, positions=pos, q_norms=qn, k_norms=kn, modulated=modulated, norm=kind)
    mod = draw((B, 2, layers, 3, C), seed, 50, 0.4) if modulated else None
    return chain, draw((B, N, C), seed, 60), mod


def rows_of(segs, live):
    idx, at = [], 0
    for k, n in segs:
        if (k in (rc.SEG_TEXT, rc.SEG_TARGET)) == live:
            idx += range(at, at + n)
        at += n
    return idx


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("H,D", [(2, 64), (2, 128)])
def test_cached_rows_equal_the_recompute(H, D, kind):
    segs = [(0, 64), (1, 128), (2, 256), (3, 192), (3, 64)]
    chain, h, mod = make(segs, "paper", 2, H, D, 2, seed=3, kind=kind)
    live, static = rows_of(segs, True), rows_of(segs, False)
    per_layer = []
    full = chain.full(h, modulation=mod, collect=per_layer, last_round_split=False)
    caches = chain.prefill(h[:, static].contiguous(), modulation=mod[:, 1:].contiguous())
    steps = []
    out = chain.step(h[:, live].contiguous(), caches, modulation=mod[:, :1].contiguous(), splits=1, collect=steps)
    assert torch.equal(out, full[:, live])
    for a, b in zip(steps, per_layer):
        assert torch.equal(a, b[:, live])


def test_plain_chain_with_rotation_only():
    segs = [(0, 64), (1, 64), (2, 128), (3, 64)]
    chain, h, _ = make(segs, "perref", 1, 2, 128, 2, seed=5, modulated=False, norms=False, interleaved=False)
    live, static = rows_of(segs, True), rows_of(segs, False)
    full = chain.full(h, last_round_split=False)
    caches = chain.prefill(h[:, static].contiguous())
    assert torch.equal(chain.step(h[:, live].contiguous(), caches, splits=1), full[:, live])
    base = rc.Chain(chain.layout, chain.w_qkv, chain.w_o, 2, 128)
    assert not torch.equal(base.full(h, last_round_split=False), full)  # positions matter


def test_refused_modulation():
    segs = [(1, 64), (2, 64), (3, 64)]
    chain, h, mod = make(segs, "paper", 1, 2, 64, 1, seed=6)
    with pytest.raises(ValueError, match="modulation must be"):
        chain.full(h)
    with pytest.raises(ValueError, match="modulation must be"):
        chain.full(h, modulation=mod[:, :1])
    plain = rc.Chain(chain.layout, chain.w_qkv, chain.w_o, 2, 64)
    with pytest.raises(ValueError, match="modulated=True"):
        plain.full(h, modulation=mod)


def reference(chain, h, mod, dh):
    """The chain in 64 bits, and its gradients by differentiation."""
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    H, D, C = chain.H, chain.D, chain.C
    x = h if h.requires_grad else leaf(h)
    wq, wo = [leaf(w) for w in chain.w_qkv], [leaf(w) for w in chain.w_o]
    qn = [leaf(w) for w in chain.q_norms] if chain.q_norms else None
    kn = [leaf(w) for w in chain.k_norms] if chain.k_norms else None
    m = leaf(mod) if mod is not None else None
    segs = chain.layout.segments
    lens = torch.tensor([n for _, n in segs])
    ids = torch.repeat_interleave(torch.arange(len(segs)), lens)
    seen = torch.tensor(chain.layout.visible)[ids][:, ids].to(DEV)
    group = torch.repeat_interleave(torch.tensor([0 if k in (1, 2) else 1 for k, _ in segs]), lens).to(DEV)
    B, N = h.shape[:2]

    def norm(t):
        t = t - t.mean(-1, keepdim=True) if chain.norm == "layer" else t
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + chain.eps)

    if chain.rotary is not None:
        ang, axes = [], chain.rotary.axes
        pos = chain._positions[rc.ROWS_ALL].double()
        for a, d in enumerate(axes):
            ang += [pos[:, a] * 10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
        ang = torch.stack(ang, -1)[None, :, None]

    def turn(t, w):
        if w is not None:
            t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + chain.eps) * w
        half = ang.shape[-1]
        u, rest = t[..., :2 * half], t[..., 2 * half:]
        inter = bool(chain.rotary.c.interleaved)
        a, b = (u[..., 0::2], u[..., 1::2]) if inter else (u[..., :half], u[..., half:])
        c, s = ang.cos(), ang.sin()
        p, q = a * c - b * s, a * s + b * c
        return torch.cat([torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1), rest], -1)

    y = x
    for l in range(chain.layers):
        if m is not None:
            y = norm(x) * (1 + m[:, group, l, 1]) + m[:, group, l, 0]
        qkv = (y @ wq[l].t()).view(B, N, 3, H, D)
        q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        if chain.rotary is not None:
            q, k = turn(q, qn[l] if qn else None), turn(k, kn[l] if kn else None)
        s = torch.einsum("bnhd,bmhd->bhnm", q, k) * chain.scale
        p = torch.softmax(s.masked_fill(~seen, float("-inf")), -1)
        a = torch.einsum("bhnm,bmhd->bnhd", p, v).reshape(B, N, C) @ wo[l].t()
        x = x + (a if m is None else m[:, group, l, 2] * a)
        y = x
    leaves = [x0 for x0 in [*wq, *wo, *(qn or []), *(kn or []), *([m] if m is not None else [])]]
    return x, None, leaves, (wq, wo, qn, kn, m)


@pytest.mark.parametrize("B,H,D,mask,modulated,norms,kind", [
    (1, 2, 64, "perref", True, True, "layer"), (2, 2, 64, "paper", True, False, "rms"),
    (1, 2, 128, "paper", False, True, "layer"), (1, 4, 64, "dense", False, False, "layer")])
def test_gradient_of_the_chain(B, H, D, mask, modulated, norms, kind):
    segs = [(0, 17), (1, 40), (2, 130), (3, 70), (3, 33)]
    chain, h, mod = make(segs, mask, B, H, D, 2, seed=7, modulated=modulated, norms=norms, kind=kind, interleaved=D == 64)
    dh = draw(h.shape, 7, 70)
    got = chain.full_backward(h, dh, modulation=mod)

    x = h.double().requires_grad_()
    out, _, leaves, (wq, wo, qn, kn, m) = reference(chain, x, mod, dh)
    grads = torch.autograd.grad(out, [x] + leaves, dh.double())
    it = iter(grads)

    def near(name, g, ref):
        rel = ((g.double() - ref).norm() / ref.norm()).item()
        print(f"[chain grad] {name} rel_l2={rel:.2e}", flush=True)
        assert g.shape == ref.shape and rel <= REL, (name, rel)

    near("h", got.h, next(it))
    for name, lst in (("w_qkv", got.w_qkv), ("w_o", got.w_o), ("q_norms", got.q_norms), ("k_norms", got.k_norms)):
        if lst is not None:
            for l, g in enumerate(lst):
                near(f"{name}[{l}]", g, next(it))
    if m is not None:
        ref = next(it)
        near("modulation", got.modulation, ref)
    # on another stream: the same bits
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    again = chain.full_backward(h, dh, modulation=mod, stream=s)
    s.synchronize()
    assert torch.equal(again.h, got.h) and torch.equal(again.w_qkv[0], got.w_qkv[0])


def test_chain_captured_and_replayed():
    """A cached step and the gradient of the recompute, each captured once and
    replayed with eager work of the same chain in between; two graphs and the
    eager calls share nothing but inputs."""
    segs = [(0, 17), (1, 40), (2, 130), (3, 70)]
    chain, h, mod = make(segs, "perref", 1, 2, 64, 2, seed=9)
    live, static = rows_of(segs, True), rows_of(segs, False)
    h_live, h_static, dh = h[:, live].contiguous(), h[:, static].contiguous(), draw(h.shape, 9, 71)
    m_live, m_static = mod[:, :1].contiguous(), mod[:, 1:].contiguous()
    flat = lambda g: [g.h, *g.w_qkv, *g.w_o, *g.q_norms, *g.k_norms, g.modulation]  # noqa: E731

    def eager():
        caches = chain.prefill(h_static, modulation=m_static)
        return caches, chain.step(h_live, caches, modulation=m_live), chain.full_backward(h, dh, modulation=mod)

    caches, step, grads = eager()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        step_out = chain.step(h_live, caches, modulation=m_live)
    with torch.cuda.graph(graphs[1]):
        grads_out = chain.full_backward(h, dh, modulation=mod)
    for i in range(3):
        for t in [step_out, *flat(grads_out)]:
            t.fill_(float("nan"))
        for g in graphs if i % 2 else reversed(graphs):
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(step_out, step)
        for a, b in zip(flat(grads_out), flat(grads)):
            assert torch.equal(a, b)
        eager()
