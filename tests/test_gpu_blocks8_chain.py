"""Chains whose projections and checkpoints are in 8 bits.

Exactness: a row's codes and its product's bits depend on the row alone, so the
cached path's live rows equal the recompute's bit for bit, as in bf16.

Gradient: against the chain in 64 bits over the same 8-bit weights, its activations
rounded where the library rounds them and differentiated straight through that.
A rounding to e4m3 is off by 2^-4 / sqrt(3) = 3.6e-2 of the value in the root mean
square, independent of the others.  linear="fp8": a layer's gradient passes two such
roundings (of dy before each inputs' gradient): 3.6e-2 sqrt(4) = 7.2e-2 for two
layers; the four roundings of activations are those of the reference but for values
within bf16's 2^-8 of a border, 2^-4 sqrt(2 * 2^-8 / 2^-4) = 2.2e-2 each; with bf16's own
1.4e-2 together sqrt(7.2^2 + 4.4^2 + 1.4^2) 1e-2 = 8.6e-2, carried with a gain of the
order of one: 1.5e-1 of a gradient's L2 norm is allowed.  checkpoints="fp8": one
rounding of each value that a gradient reads, and two of the norms' rows and
branches on a path through two layers: 3.6e-2 sqrt(3) = 6.2e-2: 1.2e-1 is allowed, both together
2e-1."""
import pytest
import torch

import paper_2608_21229_amd as rc
from tests import blocks8_plain as plain
from tests.test_gpu_layer_chain import draw, make, reference, rows_of

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SEGS = [(0, 17), (1, 40), (2, 130), (3, 70), (3, 33)]


def chain8(base, linear="fp8", checkpoints="bf16"):
    """The chain of make() with 8-bit projections or checkpoints."""
    return rc.Chain(base.layout, base.w_qkv, base.w_o, base.H, base.D, rotary=base.rotary,
                    positions=base._positions[rc.ROWS_ALL] if base.rotary else None, q_norms=base.q_norms,
                    k_norms=base.k_norms, modulated=base.modulated, norm=base.norm, linear=linear, checkpoints=checkpoints)


def flat(g):
    return [g.h, *g.w_qkv, *g.w_o, *(g.q_norms or []), *(g.k_norms or []), *([] if g.modulation is None else [g.modulation])]


@pytest.mark.parametrize("H,D", [(2, 64), (3, 64), (2, 128)])
def test_cached_rows_equal_the_recompute(H, D):
    segs = [(0, 64), (1, 128), (2, 256), (3, 192), (3, 64)]
    base, h, mod = make(segs, "paper", 2, H, D, 2, seed=3)
    chain = chain8(base)
    live, static = rows_of(segs, True), rows_of(segs, False)
    full = chain.full(h, modulation=mod, last_round_split=False)
    caches = chain.prefill(h[:, static].contiguous(), modulation=mod[:, 1:].contiguous())
    out = chain.step(h[:, live].contiguous(), caches, modulation=mod[:, :1].contiguous(), splits=1)
    assert torch.equal(out, full[:, live])
    if H * D % 128:  # widths that the bf16 projection does not take
        return
    off = (full - base.full(h, modulation=mod, last_round_split=False)).float().norm() / full.float().norm()
    assert 0 < off < 0.1  # two roundings per product, four products, beside the residual


def test_plain_layer_by_its_parts():
    """One layer without norms: the projections are the operators' products, and the
    gradients theirs."""
    base, h, _ = make(SEGS, "perref", 1, 2, 64, 1, seed=4, modulated=False, rotary=False, norms=False)
    chain, (M, C) = chain8(base), (h.shape[1], 128)
    x8 = rc.quantize_blocks(h.view(M, C))
    w8, o8w = (rc.quantize_blocks(w[0], square=True, transposed=True) for w in (base.w_qkv, base.w_o))
    qkv = rc.linear_fp8(x8, w8).view(1, M, 3, 2, 64)
    q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
    o, lse = rc.full_attention(chain.layout, q, k, v, want_lse=True)
    o8 = rc.quantize_blocks(o.view(M, C))
    assert torch.equal(chain.full(h).view(M, C), rc.linear_fp8(o8, o8w, residual=h.view(M, C)))
    dh = draw(h.shape, 4, 70)
    got = chain.full_backward(h, dh)
    do, dwo = rc.linear_fp8_backward(dh.view(M, C), o8, o8w)
    dq, dk, dv = rc.full_attention_backward(chain.layout, q, k, v, o, lse, do.view(o.shape))
    dqkv = torch.stack([dq, dk, dv], 2).view(M, 3 * C)
    dx, dwq = rc.linear_fp8_backward(dqkv, x8, w8, residual=dh.view(M, C))
    assert torch.equal(got.w_o[0], dwo) and torch.equal(got.w_qkv[0], dwq) and torch.equal(got.h.view(M, C), dx)


class Through(torch.autograd.Function):
    """e4m3 blocks of 128 of the bf16 rounding, differentiated as if they were not there."""

    @staticmethod
    def forward(ctx, x):
        return plain.quantize(x.reshape(-1, x.shape[-1]).bfloat16())[2].view(x.shape).to(x.device)

    @staticmethod
    def backward(ctx, g):
        return g


@pytest.mark.parametrize("linear,checkpoints,rel", [("fp8", "bf16", 1.5e-1), ("bf16", "fp8", 1.2e-1), ("fp8", "fp8", 2e-1)])
@pytest.mark.parametrize("B,H,D,mask,modulated,norms", [
    (1, 2, 64, "perref", True, True), (2, 2, 64, "paper", True, False), (1, 2, 128, "paper", False, True),
    (1, 4, 64, "dense", False, False)])
def test_gradient_of_the_chain(B, H, D, mask, modulated, norms, linear, checkpoints, rel, monkeypatch):
    base, h, mod = make(SEGS, mask, B, H, D, 2, seed=7, modulated=modulated, norms=norms)
    chain = chain8(base, linear, checkpoints)
    dh = draw(h.shape, 7, 70)
    got = chain.full_backward(h, dh, modulation=mod)

    x = h.double().requires_grad_()
    if linear == "fp8":  # the same weights' values, and activations rounded on the way
        base.w_qkv, base.w_o = ([rc.dequantize_blocks(rc.quantize_blocks(w, square=True)) for w in ws]
                                for ws in (base.w_qkv, base.w_o))
        rmatmul = torch.Tensor.__matmul__
        monkeypatch.setattr(torch.Tensor, "__matmul__",
                            lambda a, b: rmatmul(Through.apply(a), b) if b.dim() == 2 and a.dim() == 3 else rmatmul(a, b))
    out, _, leaves, _ = reference(base, x, mod, dh)
    monkeypatch.undo()
    for i, (g, ref) in enumerate(zip(flat(got), torch.autograd.grad(out, [x] + leaves, dh.double()))):
        off = ((g.double() - ref).norm() / ref.norm()).item()
        print(f"[chain8 grad] {i} rel_l2={off:.2e}", flush=True)
        assert g.shape == ref.shape and off <= rel, (i, off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    again = chain.full_backward(h, dh, modulation=mod, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat(again), flat(got)))


def test_captured_replayed_and_updated_weights():
    """The gradient captured once and replayed with eager work between; new weights
    reach replays after update_weights."""
    base, h, mod = make(SEGS, "perref", 1, 2, 64, 2, seed=9)
    chain = chain8(base, "fp8", "fp8")
    dh = draw(h.shape, 9, 71)
    want = chain.full_backward(h, dh, modulation=mod)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = chain.full_backward(h, dh, modulation=mod)
    for i in range(3):
        for t in flat(held):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(held), flat(want)))
        chain.full(h, modulation=mod)
    for w in base.w_qkv + base.w_o:
        w.mul_(-0.75)
    chain.update_weights()
    graph.replay()
    torch.cuda.synchronize()
    want = chain8(base, "fp8", "fp8").full_backward(h, dh, modulation=mod)
    assert all(torch.equal(a, b) for a, b in zip(flat(held), flat(want)))


def test_what_stays_of_a_bf16_chain():
    """Without the options nothing changes, and the option is refused where it is none."""
    base, h, mod = make(SEGS, "paper", 1, 2, 64, 1, seed=10)
    same = chain8(base, "bf16", "bf16")
    assert torch.equal(same.full(h, modulation=mod), base.full(h, modulation=mod))
    with pytest.raises(ValueError, match="linear='fp8'"):
        same.update_weights()
    for bad in (dict(linear="int8"), dict(checkpoints="fp4")):
        with pytest.raises(ValueError, match="must be 'bf16' or 'fp8'"):
            chain8(base, **bad)
