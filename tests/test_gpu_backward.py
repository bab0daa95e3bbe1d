"""The gradient of the full recompute against its formula in 64 bits.

Bounds.  A kernel's p_ij and ds_ij are rounded once to bf16 (half a step:
u = 2^-8 relative) before they enter a product, and the result once:
    |dv - ref| <= u (sum_i p |do| + |dv|)
    |dq - ref| <= u (scale sum_j |ds| |k| + |dq|), dk alike with q
up to second order and to fp32 arithmetic.  The latter: p = 2^x with x off by
a few 2^-24 of the terms of x (logits and lse up to 2^6 here, so 2^-17
relative), and do.v - D off by at most 2 D 2^-24 <= 2^-16 of sum |do| |v| and
of sum |do| |o|.  Each of these is multiplied out below with 2^-15."""
import pytest
import torch

import paper_2608_21229_amd as rc
from synthgen import bf16_normal, derive_seed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, F = 2.0 ** -8, 2.0 ** -15


def _visible(L):
    lens = torch.tensor([n for _, n in L.segments])
    ids = torch.repeat_interleave(torch.arange(len(lens)), lens)
    return torch.tensor(L.visible)[ids][:, ids]


def _inputs(L, B, H, D, seed, std=1.0, fused=False, dlse=False):
    N = sum(n for _, n in L.segments)
    draw = lambda i, s=1.0: bf16_normal((B, N, H, D), derive_seed(seed, 0, 0, i), s).to(DEV)  # noqa: E731
    q, k, v = draw(0, std), draw(1, std), draw(2)
    if fused:
        buf = torch.stack((q, k, v), 2)
        q, k, v = buf[:, :, 0], buf[:, :, 1], buf[:, :, 2]
    o, lse = rc.full_attention(L, q, k, v, want_lse=True)
    g = torch.Generator().manual_seed(seed + 77)
    dl = torch.randn(B, H, N, generator=g).to(DEV) if dlse else None
    return q, k, v, o, lse, draw(3), dl


def _reference(L, q, k, v, o, lse, do, dlse, scale):
    """Gradients in 64 bits and the bounds of their errors."""
    B, N, H, D = q.shape
    seen = _visible(L).to(q.device)
    ref = [torch.zeros(B, N, H, D, dtype=torch.float64, device=q.device) for _ in range(3)]
    tol = [torch.zeros_like(r) for r in ref]
    for b in range(B):
        for h in range(H):
            Q, K, V, O, G = (t[b, :, h].double() for t in (q, k, v, o, do))
            none = ~seen.any(1)
            O, G = O.masked_fill(none[:, None], 0), G.masked_fill(none[:, None], 0)
            p = torch.where(seen, torch.exp(scale * (Q @ K.t()) - lse[b, h].double()[:, None]), 0.0)
            d = (O * G).sum(1) - (dlse[b, h].double() if dlse is not None else 0.0)
            ds = torch.where(seen, p * (G @ V.t() - d[:, None]), 0.0)
            size = p * (G.abs() @ V.abs().t() + (O.abs() * G.abs()).sum(1)[:, None] + 1.0)
            for i, (r, bound, small) in enumerate((
                    (scale * ds @ K, scale * ds.abs() @ K.abs(), scale * size @ K.abs()),
                    (scale * ds.t() @ Q, scale * ds.abs().t() @ Q.abs(), scale * size.t() @ Q.abs()),
                    (p.t() @ G, p.t() @ G.abs(), p.t() @ G.abs()))):
                ref[i][b, :, h] = r
                tol[i][b, :, h] = U * (bound + r.abs()) + F * small + 1e-30
    return ref, tol


def _check(L, B, H, D, seed, std=1.0, fused=False, dlse=False, scale=None):
    q, k, v, o, lse, do, dl = _inputs(L, B, H, D, seed, std, fused, dlse)
    if scale is not None:
        o, lse = rc.full_attention(L, q, k, v, scale=scale, want_lse=True)
    got = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl, scale=scale)
    ref, tol = _reference(L, q, k, v, o, lse, do, dl, D ** -0.5 if scale is None else scale)
    for name, g, r, t in zip(("dq", "dk", "dv"), got, ref, tol):
        assert torch.isfinite(g).all(), name
        over = ((g.double() - r).abs() / t).max().item()
        print(f"[grad] {name} B={B} H={H} D={D} err/bound={over:.3f}", flush=True)
        assert over <= 1.0, (name, over)
    return (q, k, v, o, lse, do, dl), got


PRESETS = ["perref", "paper", "isolated", "dense"]
SMALL = [(0, 8), (1, 16), (2, 64), (3, 64)]
EDGES = [(0, 1), (1, 33), (2, 257), (3, 63), (3, 65), (3, 1)]
LONG = [(0, 37), (1, 130), (2, 700), (3, 512), (3, 301)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("segs", [SMALL, EDGES, LONG], ids=["small", "edges", "long"])
@pytest.mark.parametrize("preset", PRESETS)
def test_gradient_of_presets(preset, segs, D):
    _check(rc.Layout(segs, preset), 1, 2, D, seed=3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 255, 256, 257, 320])
def test_gradient_of_one_segment(n, D):
    _check(rc.Layout([(2, n)], "dense"), 1, 1, D, seed=n)


@pytest.mark.parametrize("D", [64, 128])
def test_gradient_of_random_masks(D):
    g = torch.Generator().manual_seed(5)
    for i in range(8):
        n = 2 + i
        segs = [(int(torch.randint(0, 4, (1,), generator=g)), int(torch.randint(1, 150, (1,), generator=g)))
                for _ in range(n)]
        mask = (torch.rand(n, n, generator=g) < 0.5).tolist()
        _check(rc.Layout(segs, mask), 2, 2, D, seed=20 + i, fused=bool(i % 2), dlse=bool(i % 3))


@pytest.mark.parametrize("std", [0.05, 2.0])
def test_gradient_of_flat_and_sharp_softmax(std):
    _check(rc.Layout(LONG, "paper"), 1, 2, 128, seed=9, std=std)


def test_gradient_with_another_scale():
    _check(rc.Layout(LONG, "perref"), 2, 1, 64, seed=10, scale=0.31, dlse=True)


def test_fused_buffers_and_strides():
    """Q/K/V and the gradients as views of fused buffers give the bits of separate ones."""
    L = rc.Layout(EDGES, "perref")
    (q, k, v, o, lse, do, dl), got = _check(L, 2, 3, 128, seed=11, fused=True, dlse=True)
    B, N, H, D = q.shape
    buf = torch.full((B, N, 3, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    views = [buf[:, :, i] for i in range(3)]
    ws = torch.full((L.backward_workspace_bytes(B, H, D) // 4,), float("nan"), device=DEV)
    out = rc.full_attention_backward(L, q.contiguous(), k.contiguous(), v.contiguous(), o, lse, do, dlse=dl,
                                     dq=views[0], dk=views[1], dv=views[2], workspace=ws)
    for a, b, c in zip(out, got, views):
        assert a is c and torch.equal(a, b)


def test_rows_that_read_nothing_and_keys_nobody_reads():
    L = rc.Layout([(0, 40), (1, 20), (2, 90), (3, 70)], "isolated")
    q, k, v, o, lse, do, dl = _inputs(L, 1, 2, 128, 13, dlse=True)
    assert torch.isinf(lse[:, :, :40]).all()
    ref = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    for g in ref:
        assert (g[:, :40] == 0).all() and (g[:, 40:] != 0).any()
    # what the anchors' rows hold does not matter
    for t in (q, k, v, o, do):
        t[:, :40] = float("nan")
    dl[:, :, :40] = float("nan")
    for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl), ref):
        assert torch.equal(a[:, 40:], b[:, 40:])


def test_repeats_are_the_same_bits():
    L = rc.Layout(LONG, "perref")
    q, k, v, o, lse, do, dl = _inputs(L, 2, 3, 128, 17, dlse=True)
    both = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    again = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    for a, b in zip(both, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("segs,preset,H", [([(2, 1000)], "dense", 1), ([(0, 37), (1, 130), (2, 1700), (3, 1512), (3, 301)], "paper", 1),
                                           ([(0, 64), (1, 33), (2, 2500), (3, 700)], "perref", 2),
                                           ([(0, 300), (1, 1), (2, 3000), (3, 65), (3, 1)], "isolated", 1)])
def test_few_heads_split_the_streamed_rows(segs, preset, H, D):
    """Few work-groups: their streamed rows are cut into pieces, whose fp32 sums are merged."""
    L = rc.Layout(segs, preset)
    N = sum(n for _, n in segs)
    assert L.backward_workspace_bytes(1, H, D) > 2 * (H * N * 4 + 16), "no pieces"
    (q, k, v, o, lse, do, dl), got = _check(L, 1, H, D, seed=37, fused=True, dlse=True)
    ws = torch.full((L.backward_workspace_bytes(1, H, D) // 4 + 1,), float("nan"), device=DEV)
    for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl, workspace=ws), got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("preset", ["perref", "paper"])
def test_many_work_groups(preset, D):
    """More work-groups than CUs, whose rings wrap many times: against the formula, and the same bits in every pass."""
    L = rc.Layout([(0, 37), (1, 203), (2, 1577), (3, 1024), (3, 519)], preset)
    (q, k, v, o, lse, do, dl), got = _check(L, 1, 24, D, seed=31, fused=True, dlse=True)
    for _ in range(4):
        for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl), got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("segs,preset", [([(2, n)], "dense") for n in (129, 160, 191, 193, 224, 255, 256, 257, 320, 513)] +
                         [([(0, 257), (1, 33), (2, 300), (3, 255), (3, 1)], p) for p in PRESETS],
                         ids=lambda x: x if isinstance(x, str) else "-".join(str(n) for _, n in x))
def test_many_heads_take_large_own_tiles(segs, preset, D):
    """Enough heads that own tiles of 256 rows are chosen (as the planner's host test asserts): some of the
    heads against the formula, all of them the same bits again and in strided outputs."""
    L, B, H = rc.Layout(segs, preset), 2, 128
    q, k, v, o, lse, do, dl = _inputs(L, B, H, D, seed=41, dlse=True)
    got = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    pick = [0, 51, 127]
    ref, tol = _reference(L, *(t[:, :, pick] for t in (q, k, v, o)), lse[:, pick], do[:, :, pick], dl[:, pick], D ** -0.5)
    for name, g, r, t in zip(("dq", "dk", "dv"), got, ref, tol):
        assert torch.isfinite(g).all(), name
        over = ((g[:, :, pick].double() - r).abs() / t).max().item()
        assert over <= 1.0, (name, over)
    buf = torch.full((B, q.shape[1], 3, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, *buf.unbind(2), dlse=dl), got):
        assert torch.equal(a, b)


def test_finite_differences():
    """sum(w O) + sum(u lse) along random directions, in 64 bits, against the kernel's gradient of them."""
    L = rc.Layout([(0, 5), (1, 40), (2, 70), (3, 33)], "paper")
    q, k, v, o, lse, do, dl = _inputs(L, 1, 1, 64, 19, dlse=True)
    got = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    seen = _visible(L).to(DEV)

    def value(Q, K, V):
        s = (Q @ K.t() / 8.0).masked_fill(~seen, float("-inf"))
        return ((torch.softmax(s, 1) @ V) * do[0, :, 0].double()).sum() + (torch.logsumexp(s, 1) * dl[0, 0].double()).sum()

    at = [t[0, :, 0].double() for t in (q, k, v)]
    g = torch.Generator().manual_seed(1)
    for i in range(3):
        step = torch.randn(at[0].shape, generator=g, dtype=torch.float64).to(DEV)
        eps = 1e-4
        diff = (value(*[a + eps * step * (i == j) for j, a in enumerate(at)])
                - value(*[a - eps * step * (i == j) for j, a in enumerate(at)])) / (2 * eps)
        along = (got[i][0, :, 0].double() * step).sum()
        # rounding: u per element and product, random in sign; |got| |step| as its scale
        scale = (got[i][0, :, 0].double().norm() * step.abs().max()).item()
        assert abs((along - diff).item()) <= 4 * U * scale, (i, along.item(), diff.item())


def test_captured_and_replayed():
    L = rc.Layout(SMALL, "perref")
    q, k, v, o, lse, do, _ = _inputs(L, 1, 2, 128, 23)
    outs = [torch.zeros_like(o) for _ in range(3)]
    ws = torch.empty(L.backward_workspace_bytes(1, 2, 128), dtype=torch.uint8, device=DEV)
    ref = rc.full_attention_backward(L, q, k, v, o, lse, do)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        rc.full_attention_backward(L, q, k, v, o, lse, do, *outs, workspace=ws)
    for i in range(3):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, ref):
            assert torch.equal(a, b)
        rc.full_attention_backward(L, q, k, v, o, lse, do)


def test_on_another_stream():
    L = rc.Layout(LONG, "perref")
    q, k, v, o, lse, do, _ = _inputs(L, 1, 2, 64, 29)
    ref = rc.full_attention_backward(L, q, k, v, o, lse, do)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = rc.full_attention_backward(L, q, k, v, o, lse, do, stream=s)
    s.synchronize()
    for a, b in zip(out, ref):
        assert torch.equal(a, b)
