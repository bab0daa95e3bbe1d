"""The layer operators on views whose rows lie more than 2^32 bytes apart (one
5 GB buffer with 4 Mi elements per row holds every operand side by side): the
same bits as on contiguous tensors."""
import pytest
import torch

import paper_2608_21229_amd as rc
from synthgen import bf16_normal, derive_seed

pytestmark = pytest.mark.gpu

DEV, N, LD = "cuda:0", 600, 1 << 22


@pytest.fixture(scope="module")
def wide():
    buf = torch.empty(1, N, LD, dtype=torch.bfloat16, device=DEV)
    assert (N - 1) * LD * 2 > 1 << 32
    yield buf
    del buf
    torch.cuda.empty_cache()


def column(buf, at, t):
    """A view of t's shape in the buffer's columns [at, at + t[0, 0].numel()), holding t."""
    view = buf[:, :, at:at + t[0, 0].numel()].view(t.shape)
    return view.copy_(t)


def draw(shape, i, std=1.0):
    return bf16_normal(tuple(shape), derive_seed(31, 0, 0, i), std).to(DEV)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_gradient(wide, D):
    L = rc.Layout([(0, 40), (1, 60), (2, 300), (3, 200)], "perref")
    q, k, v, do = (draw((1, N, 2, D), i) for i in range(4))
    o, lse = rc.full_attention(L, q, k, v, want_lse=True)
    ref = rc.full_attention_backward(L, q, k, v, o, lse, do)
    views = [column(wide, 4096 * (1 + i), t) for i, t in enumerate((q, k, v, *(torch.zeros_like(q) for _ in range(3))))]
    got = rc.full_attention_backward(L, *views[:3], o, lse, do, *views[3:])
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


def test_rotation(wide):
    R = rc.Rotary(128, (16, 56, 56))
    q, k, dq, dk = (draw((1, N, 3, 128), 10 + i) for i in range(4))
    w = 1 + draw((128,), 14, 0.2)
    pos = torch.arange(3 * N, dtype=torch.int32, device=DEV).view(N, 3)
    ref = rc.qk_rotary(R, q, k, pos, q_norm=w, k_norm=w)
    back = rc.qk_rotary_backward(R, dq, dk, pos, q=q, k=k, q_norm=w, k_norm=w)
    vq, vk, vdq, vdk = (column(wide, 4096 * (1 + i), t) for i, t in enumerate((q, k, dq, dk)))
    got = rc.qk_rotary_backward(R, vdq, vdk, pos, q=vq, k=vk, q_norm=w, k_norm=w, dq_out=vdq, dk_out=vdk)
    for a, b in zip(got, back):
        assert torch.equal(a, b)
    for a, b in zip(rc.qk_rotary(R, vq, vk, pos, q_norm=w, k_norm=w, q_out=vq, k_out=vk), ref):
        assert torch.equal(a, b)


def test_gated_norm(wide):
    C = 1160
    h, x, dy, dh = (draw((1, N, C), 20 + i) for i in range(4))
    gate, scale, shift = draw((1, 2, 3 * C), 24).chunk(3, -1)
    args = dict(gate=gate, scale=scale, shift=shift, spans=[(N - 101, 1), (101, 0)])
    ref = rc.gated_norm(h, x, **args)
    back = rc.gated_norm_backward(dy, ref[0], x, dh=dh, **args)
    vh, vx, vy, vdy, vdh = (column(wide, 4096 * (1 + i), t) for i, t in enumerate((h, x, h, dy, dh)))
    got = rc.gated_norm(vh, vx, h_out=vh, y=vy, **args)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    for a, b in zip(rc.gated_norm_backward(vdy, vh, vx, dh=vdh, dh_out=vdh, dx=vx, **args), back):
        assert (a is None and b is None) or torch.equal(a, b)
