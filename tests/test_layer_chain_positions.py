"""The positions that a chain is given are its own from then on: later writes
to the caller's tensor reach neither the recompute nor the cached path."""
import pytest
import torch

import paper_2608_21229_amd as rc

SEGS = [(0, 64), (1, 64), (2, 128), (3, 64)]
H, D = 2, 64
N = sum(n for _, n in SEGS)


def make(dev, positions, norms=True):
    g = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(dev)  # noqa: E731
    C = H * D
    w_qkv, w_o = [rn(3 * C, C) * C ** -0.5 for _ in range(2)], [rn(C, C) * C ** -0.5 for _ in range(2)]
    w = [1 + rn(D) * 0.2 for _ in range(2)] if norms else None
    return rc.Chain(rc.Layout(SEGS, "perref"), w_qkv, w_o, H, D, rotary=rc.Rotary(D, (16, 24, 24)), positions=positions,
                    q_norms=w, k_norms=w), rn(1, N, C)


def grid(dev):
    return torch.arange(3 * N, dtype=torch.int32).view(N, 3).remainder(61).to(dev)


def test_the_chain_holds_a_copy():
    for positions in (grid("cpu"), grid("cpu").t().contiguous().t(), grid("cpu").repeat(1, 2)[:, :3]):
        chain, _ = make("cpu", positions)
        held = [t for t in chain._positions.values()]
        before = [t.clone() for t in held]
        positions.fill_(7)
        assert len(held) == 3 and all(t.is_contiguous() for t in held)
        for a, b in zip(held, before):
            assert torch.equal(a, b)
        assert torch.equal(chain._positions[rc.ROWS_ALL], grid("cpu"))


def rows(live):
    at, out = 0, []
    for k, n in SEGS:
        if (k in (1, 2)) == live:
            out += range(at, at + n)
        at += n
    return out


@pytest.mark.gpu
def test_writes_to_the_callers_positions_change_nothing():
    positions = grid("cuda")
    chain, h = make("cuda", positions)
    full, grads = chain.full(h, last_round_split=False), chain.full_backward(h, h)
    positions.fill_(1000)
    assert torch.equal(chain.full(h, last_round_split=False), full)
    again = chain.full_backward(h, h)
    assert torch.equal(again.h, grads.h) and torch.equal(again.q_norms[0], grads.q_norms[0])
    caches = chain.prefill(h[:, rows(False)].contiguous())
    assert torch.equal(chain.step(h[:, rows(True)].contiguous(), caches, splits=1), full[:, rows(True)])


@pytest.mark.gpu
def test_positions_that_are_not_contiguous():
    wide = torch.zeros(N, 5, dtype=torch.int32, device="cuda")
    wide[:, 1:4] = grid("cuda")
    (a, h), (b, _) = make("cuda", wide[:, 1:4]), make("cuda", grid("cuda"))
    assert torch.equal(a.full(h), b.full(h)) and torch.equal(a.full_backward(h, h).h, b.full_backward(h, h).h)
