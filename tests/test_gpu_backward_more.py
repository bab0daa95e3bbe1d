"""The attention gradient where its header promises zeros, and where two of its
schedules meet.  Bounds and reference as in test_gpu_backward.py."""
import pytest
import torch

import paper_2608_21229_amd as rc
from tests.test_gpu_backward import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H", [(1, 2), (2, 128)], ids=["own128", "own256"])
def test_zeros_whatever_the_rows_hold(B, H, D):
    """Anchors that read nothing and that nobody reads, all of their operands NaN or infinite: exact zeros in
    outputs that held NaN, and the other rows' bits untouched, at both sizes of own tiles."""
    n = 257
    L = rc.Layout([(0, n), (1, 33), (2, 300), (3, 255), (3, 1)], "isolated")
    q, k, v, o, lse, do, dl = _inputs(L, B, H, D, 13, dlse=True)
    assert torch.isinf(lse[:, :, :n]).all()
    ref = rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl)
    for bad in (float("nan"), float("inf")):
        for t in (q, k, v, o, do):
            t[:, :n] = bad
        dl[:, :, :n] = bad
        outs = [torch.full_like(q, float("nan")) for _ in range(3)]
        ws = torch.full((L.backward_workspace_bytes(B, H, D) // 4,), float("nan"), device=q.device)
        for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, *outs, dlse=dl, workspace=ws), ref):
            assert (a[:, :n] == 0).all() and torch.equal(a[:, n:], b[:, n:])


PIECES = [([(0, 257), (1, 130), (2, 136)], "perref", 2, 4, 128), ([(0, 257), (1, 130), (2, 109), (3, 145)], "paper", 2, 4, 64),
          ([(0, 64), (1, 512), (2, 1024), (3, 1024), (3, 1024)], "perref", 1, 8, 128)]


@pytest.mark.parametrize("segs,preset,B,H,D", PIECES)
def test_pieces_of_whole_heads_per_xcd(segs, preset, B, H, D):
    """Heads that divide over the XCDs, few enough that tiles are cut into pieces."""
    L, N = rc.Layout(segs, preset), sum(n for _, n in segs)
    assert B * H % 8 == 0 and L.backward_workspace_bytes(B, H, D) > 2 * (B * H * N * 4 + 16), "no pieces"
    (q, k, v, o, lse, do, dl), got = _check(L, B, H, D, seed=43, fused=True, dlse=True)
    ws = torch.full((L.backward_workspace_bytes(B, H, D) // 4 + 1,), float("nan"), device=q.device)
    for a, b in zip(rc.full_attention_backward(L, q, k, v, o, lse, do, dlse=dl, workspace=ws), got):
        assert torch.equal(a, b)
    # every head and entry alone gives its rows of the whole call, to the rounding of another order of sums
    one = rc.full_attention_backward(L, q[-1:, :, 2:3], k[-1:, :, 2:3], v[-1:, :, 2:3], o[-1:, :, 2:3].contiguous(),
                                     lse[-1:, 2:3].contiguous(), do[-1:, :, 2:3].contiguous(), dlse=dl[-1:, 2:3].contiguous())
    for a, b in zip(one, got):
        b = b[-1:, :, 2:3].float()
        assert (a.float() - b).norm() <= 2.0 ** -8 * b.norm()
