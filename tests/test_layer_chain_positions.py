"""The positions that a chain is given are its own from then on: later writes
to the caller's tensor reach neither the recompute nor the cached path, and a
chain that is dropped leaves them to the streams that still read them."""
import contextlib

import pytest
import torch

import paper_2608_21229_amd as rc
from paper_2608_21229_amd import binding as rcb

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


@pytest.mark.parametrize("own", [True, False], ids=["stream", "current"])
def test_positions_are_marked_on_the_stream_that_reads_them(own, monkeypatch):
    """With stream= and under torch's own stream context alike."""
    chain, h = make("cpu", grid("cpu"))
    current, marked = ["main"], []

    @contextlib.contextmanager
    def fake_stream(s):
        current.append(s)
        yield
        current.pop()

    class Side:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "Stream", Side)
    monkeypatch.setattr(torch.cuda, "stream", fake_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: marked.append((t.data_ptr(), s)))
    monkeypatch.setattr(rcb, "_inputs", lambda q, k, v: q.device)
    monkeypatch.setattr(rcb, "_rows_view", lambda t, what: t.stride(0))
    monkeypatch.setattr(rcb, "_heads", lambda *a: None)
    monkeypatch.setattr(rcb, "_call", lambda fn, dev, stream, *a: None)
    side = Side()
    static, live = h[:, :128], h[:, :192]
    calls = {rc.ROWS_STATIC: lambda s: chain.prefill(static, stream=s),
             rc.ROWS_LIVE: lambda s: chain.step(live, chain.new_caches(1, "cpu"), stream=s),
             rc.ROWS_ALL: lambda s: chain.full(h, stream=s)}
    for which, call in list(calls.items()) + [(rc.ROWS_ALL, lambda s: chain.full_backward(h, h, stream=s))]:
        marked.clear()
        if own:
            call(side)
        else:
            with fake_stream(side):
                call(None)
        assert (chain._positions[which].data_ptr(), side) in marked


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


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["prefill", "step", "full", "full_backward"])
def test_a_dropped_chain_leaves_its_positions_to_the_stream(name):
    """The call is queued behind a delay, the chain dropped, and all memory that
    the current stream can then get overwritten before the call reads its positions."""
    def calls(chain, h):
        st, lv = h[:, rows(False)].contiguous(), h[:, rows(True)].contiguous()
        caches = chain.new_caches(1, "cuda")
        for t in [x for c in caches for x in c]:
            t.fill_(0.5)
        keep = [st, lv, caches, chain.w_qkv, chain.w_o, chain.q_norms, h]  # the caller's own tensors
        return {"prefill": lambda: [x for c in chain.prefill(st) for x in c], "step": lambda: [chain.step(lv, caches)],
                "full": lambda: [chain.full(h)], "full_backward": lambda: [chain.full_backward(h, h).h]}[name], keep

    chain, h = make("cuda", grid("cuda"))
    want = calls(chain, h)[0]()
    chain, h = make("cuda", grid("cuda"))
    call, keep = calls(chain, h)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()  # the side stream's pool holds what the call needs
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # some 50 ms
        got = call()
    del chain, call
    junk = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0x11)
            for n in (1 << p for p in range(9, 22)) for _ in range(8)]
    torch.cuda.synchronize()
    del junk, keep
    for a, b in zip(got, want):
        assert torch.equal(a, b)
