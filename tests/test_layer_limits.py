"""Sizes that each fit but whose launches do not: refused by the call, and 0
from the workspace query, before the planner adds up costs that 64 bits do not hold."""
import ctypes

import pytest

import paper_2608_21229_amd as rc

FAKE = 0x7f0000000000


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,n", [(65535, 65535, 1 << 24), (65535, 65535, 1 << 20), (65535, 65535, 1), (1, 65535, 1 << 24),
                                   (64, 128, 1 << 16)])
def test_attention_gradient_beyond_its_launches(B, H, n, D):
    L = rc.Layout([(2, n)], "dense")
    assert L.backward_workspace_bytes(B, H, D) == 0
    status = rc.lib().rc_full_attention_backward(ctypes.byref(L.c), B, H, D, 0.1, FAKE, FAKE, FAKE, 1 << 23, FAKE, FAKE, FAKE,
                                                 None, FAKE, FAKE, FAKE, 1 << 23, FAKE, 1 << 62, None)
    assert status == rc.RC_ERR_ARG and "grid limit" in rc.lib().rc_last_error().decode()


@pytest.mark.parametrize("D", [64, 128])
def test_attention_gradient_of_the_largest_sizes(D):
    """As many rows as a launch has threads for: two floats a row, and whole tiles."""
    n = 1 << 16
    B, H = 8, (1 << 32) // (8 * n * (D // 8)) - 1
    assert rc.Layout([(2, n)], "dense").backward_workspace_bytes(B, H, D) == 2 * B * H * n * 4
    assert rc.Layout([(2, 1 << 24)], "dense").backward_workspace_bytes(1, 1, D) >= 2 * 4 << 24
