"""The gated norm's gradient where a modulation is infinite: rows that a
work-group has no work for add nothing to the gradients that rows share.  What
is not finite follows from the formula; finite sums are compared by bits."""
import pytest
import torch

import paper_2608_21229_amd as rc
from synthgen import bf16_normal, derive_seed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = float("inf")


def draw(shape, i):
    return bf16_normal(tuple(shape), derive_seed(71, 0, 0, i), 1.0).to(DEV)


@pytest.mark.parametrize("C", [64, 1024, 1928, 2560, 4096, 16384])
@pytest.mark.parametrize("post", [False, True], ids=["plain", "post"])
@pytest.mark.parametrize("N", [1, 9])
@pytest.mark.parametrize("first", [True, False], ids=["first", "middle"])
def test_an_infinite_scale_in_a_chunk_that_ends_early(C, post, N, first):
    """dh of every row is infinite, NaN in that channel, and dgate where its terms' signs agree; the
    gradients of shift and scale keep their sums.  Rows and channels that a work-group has no work for
    would make NaN of all of it."""
    h, x, dy = (draw((1, N, C), i) for i in range(3))
    gate, scale, shift = (draw((1, 1, C), i) for i in range(3, 6))
    args = dict(gate=gate, scale=scale, shift=shift, norm="rms", post_norm=post, spans=[(N, 0)])
    clean = rc.gated_norm_backward(dy, h, x, **args)
    c = 1 if first else C // 2 + 3
    scale[0, 0, c] = INF
    h = h.clone()
    got = rc.gated_norm_backward(dy, h, x, **args)
    n = h.double() * torch.rsqrt(h.double().square().mean(-1, keepdim=True) + 1e-6)
    dn = dy.double() * (1 + scale.double())
    dot = (dn * n).mean(-1, keepdim=True)
    r = torch.rsqrt(h.double().square().mean(-1, keepdim=True) + 1e-6)
    dh = r * (dn - n * dot)
    xn = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 1e-6) if post else x.double()
    want = (dh * xn).sum((0, 1))
    assert N > 1 or want.isinf().sum() >= C - 1  # several rows may disagree in every sign
    assert torch.equal(got.gate[0, 0].isnan(), want.isnan())
    assert torch.equal(got.gate[0, 0].isinf(), want.isinf()) and torch.equal(got.gate[0, 0] > 0, want > 0)
    assert torch.equal(got.shift, clean.shift) and torch.equal(got.scale, clean.scale)
