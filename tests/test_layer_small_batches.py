"""Batches of no or one token each, as slices of longer ones: the binding's
strides for them, and the rotation over them.  Sizes out of range in the
rotation's workspace query."""
import ctypes

import pytest
import torch

import paper_2608_21229_amd as rc
from paper_2608_21229_amd import binding as rcb


def test_token_stride_of_no_and_one_token():
    """With one token the batch stride is the token stride; with none, or one entry, any will do."""
    t = torch.zeros(2, 5, 3, 2, 64)
    q, k = t[:, :, 0], t[:, :, 1]
    assert rcb._tok_stride(q[:, :0], k[:, :0]) == 2 * 64
    assert rcb._tok_stride(q[:, :1], k[:, 2:3]) == 5 * 3 * 2 * 64
    assert rcb._tok_stride(q[:, :1].contiguous(), k[:, 2:3].contiguous()) == 2 * 64
    assert rcb._tok_stride(q, k) == 3 * 2 * 64
    assert rcb._tok_stride(q[:1, :1], k[1:, 4:]) >= 2 * 64
    assert rcb._tok_stride(q[:1, :0], k[1:, :0]) >= 2 * 64
    assert rcb._tok_stride(torch.zeros(2, 0, 2, 64)) == 2 * 64
    for bad in ((q[:, :2],), (q[:, :1], k[:, :1].contiguous()), (q[..., ::2],), (q.transpose(2, 3),)):
        with pytest.raises(ValueError):
            rcb._tok_stride(*bad)


@pytest.mark.parametrize("B,N", [(70_000, 5), (0, 5), (-1, 5), (2, -1), (2, 1 << 31), (65_535, 1 << 48), (65_535, (1 << 63) - 1),
                                 (1, (1 << 63) - 1)])
def test_rotation_workspace_of_sizes_out_of_range(B, N):
    R = rc.Rotary(64, (16, 24, 24))
    query = rc.lib().rc_rotary_backward_workspace_bytes
    assert query(ctypes.byref(R.c), B, N) == 0
    assert query(ctypes.byref(R.c), 65_535, 30_000) == 768 * 2 * 64 * 4


@pytest.mark.gpu
def test_rotation_of_no_tokens_of_several_entries():
    R = rc.Rotary(64, (16, 24, 24))
    q = torch.empty(3, 0, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    a, b = rc.qk_rotary(R, q, q, pos, q_norm=w)
    assert a.shape == q.shape and b.shape == q.shape
    *_, dw, dw2 = rc.qk_rotary_backward(R, q, q, pos, q=q, k=q, q_norm=w, k_norm=w)
    assert (dw == 0).all() and (dw2 == 0).all()


@pytest.mark.gpu
def test_rotation_of_one_token_of_each_entry():
    R = rc.Rotary(128, (16, 56, 56))
    g = torch.Generator().manual_seed(3)
    t = torch.randn(4, 6, 3, 5, 128, generator=g).to(torch.bfloat16).cuda()
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([[5, -3, 7]], dtype=torch.int32, device="cuda")
    q, k = t[:, 2:3, 0], t[:, 2:3, 1]
    want = rc.qk_rotary(R, q.contiguous(), k.contiguous(), pos, q_norm=w)
    back = rc.qk_rotary_backward(R, q.contiguous(), k.contiguous(), pos, q=k.contiguous(), q_norm=w)
    got = rc.qk_rotary_backward(R, q, k, pos, q=k, q_norm=w)
    assert torch.equal(got[0], back[0]) and torch.equal(got[1], back[1]) and torch.equal(got[2], back[2])
    before = t.clone()
    rc.qk_rotary(R, q, k, pos, q_norm=w, q_out=q, k_out=k)
    assert torch.equal(t[:, 2:3, 0], want[0]) and torch.equal(t[:, 2:3, 1], want[1])
    before[:, 2:3, :2] = t[:, 2:3, :2]
    assert torch.equal(t, before)


@pytest.mark.gpu
def test_attention_gradient_of_one_token_of_each_entry():
    L = rc.Layout([(2, 1)], "dense")
    g = torch.Generator().manual_seed(5)
    t = torch.randn(3, 6, 5, 2, 64, generator=g).to(torch.bfloat16).cuda()
    views = [t[:, i, :1] for i in range(6)]
    q, k, v, do = (a.contiguous() for a in views[:4])
    o, lse = rc.full_attention(L, *views[:3], want_lse=True)
    want_o, want_lse = rc.full_attention(L, q, k, v, want_lse=True)
    assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
    want = rc.full_attention_backward(L, q, k, v, o, lse, do)
    after = t.clone()
    got = rc.full_attention_backward(L, *views[:3], o, lse, do, *views[3:])
    for a, b, c in zip(got, want, views[3:]):
        assert a is c and torch.equal(a, b)
    after[:, 3:, :1] = t[:, 3:, :1]
    assert torch.equal(t, after)
