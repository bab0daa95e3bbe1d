"""Host-only checks of the layer operators' C ABI (attention gradient, rotation,
gated norm): what they refuse, with which status, before any HIP call; the
tables that rc_rotary_init fills.  Pointers are fake and never dereferenced:
every call below fails validation or has nothing to do."""
import ctypes
import math
import time

import pytest
import torch

import paper_2608_21229_amd as rc
from paper_2608_21229_amd import binding

FAKE = 0x7f0000000000
SEGS = [(0, 8), (1, 16), (2, 64), (3, 64)]


def message():
    return rc.lib().rc_last_error().decode()


# ---------------------------------------------------------------- attention gradient
def bwd(L, B=1, H=2, D=128, scale=0.1, q=FAKE, k=FAKE, v=FAKE, ts=None, o=FAKE, lse=FAKE, do=FAKE, dlse=None, dq=FAKE,
        dk=FAKE, dv=FAKE, gs=None, ws=FAKE, wsb=0):
    ts = H * D if ts is None else ts
    gs = H * D if gs is None else gs
    return rc.lib().rc_full_attention_backward(ctypes.byref(L.c), B, H, D, scale, q, k, v, ts, o, lse, do, dlse, dq, dk,
                                               dv, gs, ws, wsb, None)


@pytest.mark.parametrize("bad,status", [
    (dict(B=0), "ARG"), (dict(H=0), "ARG"), (dict(H=70000), "ARG"), (dict(D=96), "UNSUPPORTED"), (dict(scale=0.0), "ARG"),
    (dict(scale=float("nan")), "ARG"), (dict(scale=float("inf")), "ARG"), (dict(q=None), "ARG"), (dict(k=FAKE + 8), "ARG"),
    (dict(v=None), "ARG"), (dict(o=None), "ARG"), (dict(o=FAKE + 2), "ARG"), (dict(do=None), "ARG"), (dict(lse=None), "ARG"),
    (dict(lse=FAKE + 2), "ARG"), (dict(dlse=FAKE + 1), "ARG"), (dict(dq=None), "ARG"), (dict(dk=None), "ARG"),
    (dict(dv=FAKE + 4), "ARG"), (dict(ts=255), "ARG"), (dict(ts=260), "ARG"), (dict(ts=(1 << 24) + 8), "ARG"),
    (dict(gs=255), "ARG"), (dict(gs=257), "ARG"), (dict(gs=(1 << 24) + 8), "ARG"),
    (dict(scale=2.0 ** -97), "UNSUPPORTED"), (dict(scale=2.0 ** -96), "WORKSPACE"),
    (dict(), "WORKSPACE"), (dict(ws=None, wsb=1 << 40), "WORKSPACE"), (dict(ws=FAKE + 4, wsb=1 << 40), "WORKSPACE")],
    ids=lambda x: "-".join(f"{k}" for k in x) if isinstance(x, dict) else x)
def test_gradient_refusals(bad, status):
    L = rc.Layout(SEGS, "perref")
    assert bwd(L, **bad) == getattr(rc, "RC_ERR_" + status), message()
    assert message()


def test_gradient_of_a_bad_layout():
    L = rc.Layout(SEGS, "perref")
    L.c.seg[1].len = 0
    assert bwd(L, wsb=1 << 40) == rc.RC_ERR_ARG
    assert L.backward_workspace_bytes(1, 2, 128) == 0
    L = rc.Layout(SEGS, "perref")
    L.c.visible[0] = 1 << 9
    assert bwd(L, wsb=1 << 40) == rc.RC_ERR_ARG


def test_gradient_of_a_mask_that_is_fragmented_from_the_keys_side():
    """Query q reads key k where bit q % 4 of k % 16 is set: 4 lists of ranges
    for the queries (30 in all), 15 for the keys (more than the table holds)."""
    n = 32
    mask = [[bool(k % 16 >> q % 4 & 1) for k in range(n)] for q in range(n)]
    L = rc.Layout([(2, 3)] * n, mask)
    assert L.work_groups(rc.ENTRY_FULL, 1, 1, 64) > 0
    assert bwd(L, wsb=1 << 40) == rc.RC_ERR_UNSUPPORTED, message()
    assert "ranges" in message()
    assert L.backward_workspace_bytes(1, 1, 64) == 0
    with pytest.raises(rc.RcError):  # the binding names the reason, too
        rc.binding._check(bwd(L))


def test_gradient_workspace():
    L = rc.Layout([(2, 5000)], "dense")
    rows = lambda bh: 2 * ((bh * 5000 * 4 + 15) // 16 * 16)  # noqa: E731
    assert L.backward_workspace_bytes(4, 64, 128) == rows(256)   # the chip is full: no pieces
    few = L.backward_workspace_bytes(1, 1, 128) - rows(1)
    assert few > 0 and few % (256 * 128 * 4) == 0
    assert L.backward_workspace_bytes(0, 1, 128) == 0 and L.backward_workspace_bytes(1, 1, 96) == 0


# ---------------------------------------------------------------- rotation
def init(D=128, axes=(16, 56, 56), theta=10000.0, interleaved=1, continuous=0, n=None):
    R = binding.rc_rotary()
    arr = (ctypes.c_int32 * max(1, len(axes)))(*axes)
    return rc.lib().rc_rotary_init(ctypes.byref(R), D, len(axes) if n is None else n, arr, theta, interleaved, continuous), R


@pytest.mark.parametrize("bad,status", [
    (dict(D=96), "UNSUPPORTED"), (dict(axes=(16, 56, 57)), "ARG"), (dict(axes=(16, 56, 58)), "ARG"), (dict(axes=(-2, 4)), "ARG"),
    (dict(n=0), "ARG"), (dict(n=9), "ARG"), (dict(theta=0.0), "ARG"), (dict(theta=float("inf")), "ARG"),
    (dict(theta=float("nan")), "ARG"), (dict(axes=(16, 56, 50), interleaved=0), "UNSUPPORTED")],
    ids=lambda x: "-".join(f"{k}" for k in x) if isinstance(x, dict) else x)
def test_rotary_init_refusals(bad, status):
    assert init(**bad)[0] == getattr(rc, "RC_ERR_" + status), message()


@pytest.mark.parametrize("continuous", [0, 1])
def test_rotary_frequencies(continuous):
    axes = (16, 56, 40)
    status, R = init(axes=axes, continuous=continuous)
    assert status == rc.RC_OK and R.width == 112
    p = 0
    for a, d in enumerate(axes):
        for i in range(d // 2):
            e = 2.0 * p / 112 if continuous else 2.0 * i / d
            assert R.axis[p] == a
            assert math.isclose(R.turns[p] * 2 * math.pi, 10000.0 ** -e, rel_tol=1e-14)
            p += 1
    assert all(R.turns[i] == 0.0 for i in range(p, 64))


def rot(R, B=1, N=4, H=2, q=FAKE, k=FAKE, ts=256, pos=FAKE, qn=None, kn=None, eps=1e-6, qo=FAKE + 4096, ko=FAKE + 4096,
        os_=256):
    return rc.lib().rc_qk_rotary(ctypes.byref(R), B, N, H, q, k, ts, pos, 0, 0, qn, kn, eps, qo, ko, os_, None)


@pytest.mark.parametrize("bad", [
    dict(B=0), dict(H=0), dict(N=-1), dict(N=1 << 31), dict(B=60000, N=60000), dict(q=None, k=None), dict(q=FAKE + 2),
    dict(ts=255), dict(ts=260), dict(ts=1 << 25), dict(os_=200), dict(pos=None), dict(pos=FAKE + 2), dict(qn=FAKE + 2),
    dict(q=None, qn=FAKE), dict(qn=FAKE, eps=-1.0), dict(qn=FAKE, eps=float("nan")), dict(qo=None), dict(ko=FAKE + 8),
    dict(qo=FAKE, os_=512)], ids=lambda x: "-".join(x))
def test_rotation_refusals(bad):
    R = init()[1]
    assert rot(R, **bad) == rc.RC_ERR_ARG, message()


def test_rotation_needs_an_initialised_description():
    assert rot(binding.rc_rotary()) == rc.RC_ERR_ARG
    R = init()[1]
    R.axis[3] = 7
    assert rot(R) == rc.RC_ERR_ARG
    R = init()[1]
    R.turns[3] = float("nan")
    assert rot(R) == rc.RC_ERR_ARG
    R = init()[1]
    R.head_dim = 96
    assert rot(R) in (rc.RC_ERR_ARG, rc.RC_ERR_UNSUPPORTED)
    assert rot(init()[1], N=0, q=None, k=None, pos=None) == rc.RC_OK  # nothing to do


def rot_bwd(R, B=1, N=4, H=2, dq=FAKE, dk=FAKE, gs=256, pos=FAKE, q=FAKE, k=FAKE, ts=256, qn=None, kn=None, eps=1e-6,
            qo=FAKE + 4096, ko=FAKE + 4096, os_=256, dqn=None, dkn=None, ws=None, wsb=0):
    return rc.lib().rc_qk_rotary_backward(ctypes.byref(R), B, N, H, dq, dk, gs, pos, 0, 0, q, k, ts, qn, kn, eps, qo, ko,
                                          os_, dqn, dkn, ws, wsb, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dq=None, dk=None), "ARG"), (dict(gs=250), "ARG"), (dict(os_=250), "ARG"), (dict(qn=FAKE, q=None), "ARG"),
    (dict(qn=FAKE, ts=250), "ARG"), (dict(dqn=FAKE), "ARG"), (dict(qn=FAKE, dqn=FAKE + 2), "ARG"), (dict(dq=FAKE, qo=FAKE, os_=512), "ARG"),
    (dict(qn=FAKE), "WORKSPACE"), (dict(kn=FAKE, ws=FAKE + 4, wsb=1 << 30), "WORKSPACE"), (dict(qn=FAKE, ws=FAKE, wsb=16), "WORKSPACE")],
    ids=lambda x: "-".join(f"{k}" for k in x) if isinstance(x, dict) else x)
def test_rotation_gradient_refusals(bad, status):
    assert rot_bwd(init()[1], **bad) == getattr(rc, "RC_ERR_" + status), message()


# ---------------------------------------------------------------- gated norm
def desc(B=2, C=64, G=2, norm=0, post=0, N=24, eps=1e-6, rs=1.0, mb=384, mg=192, spans=((16, 0), (8, 1)), n=None):
    rows, groups = zip(*spans) if spans else ((), ())
    return binding.rc_norm(B, C, G, norm, post, N, eps, rs, mb, mg, len(spans) if n is None else n,
                           binding._I32S(*rows), binding._I32S(*groups))


def norm(d, h=FAKE, ldh=64, x=FAKE, ldx=64, gate=FAKE, scale=FAKE, shift=FAKE, w=None, wp=None, ho=FAKE, ldho=64, y=FAKE, ldy=64):
    return rc.lib().rc_gated_norm(ctypes.byref(d), h, ldh, x, ldx, gate, scale, shift, w, wp, ho, ldho, y, ldy, None)


BAD_DESC = [dict(B=0), dict(B=70000), dict(N=-1), dict(N=1 << 31), dict(C=4), dict(C=60), dict(C=16392), dict(G=0), dict(norm=2),
            dict(norm=-1), dict(eps=-1e-6), dict(eps=float("nan")), dict(rs=float("inf")), dict(mb=-8), dict(mg=4), dict(mb=12),
            dict(spans=((16, 0), (7, 1))), dict(spans=((16, 0), (8, 2))), dict(spans=((16, -1), (8, 1))), dict(spans=((-8, 0), (32, 1))),
            dict(n=33), dict(n=-1)]


@pytest.mark.parametrize("bad", BAD_DESC, ids=lambda x: "-".join(x))
def test_norm_description_refusals(bad):
    d = desc(**bad)
    assert norm(d) == rc.RC_ERR_ARG, message()
    assert rc.lib().rc_gated_norm_backward_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("bad", [
    dict(h=None), dict(h=FAKE + 8), dict(ldh=63), dict(ldh=68), dict(ldh=1 << 23), dict(x=None), dict(ho=None), dict(ldx=32),
    dict(ldho=60), dict(ldho=72), dict(y=FAKE + 2), dict(ldy=8), dict(gate=FAKE + 2), dict(scale=FAKE + 8), dict(shift=FAKE + 1),
    dict(w=FAKE + 4), dict(wp=FAKE), dict(x=None, ho=None), dict(x=None, ho=None, gate=None, y=None, scale=None, shift=None),
    dict(y=None)], ids=lambda x: "-".join(x))
def test_norm_refusals(bad):
    assert norm(desc(), **bad) == rc.RC_ERR_ARG, message()


def norm_bwd(d, dy=FAKE, lddy=64, dh=FAKE, lddh=64, h=FAKE, ldh=64, x=FAKE, ldx=64, gate=FAKE, scale=FAKE, w=None, wp=None,
             dhi=FAKE, lddhi=64, dx=FAKE, lddx=64, dgate=FAKE, dscale=FAKE, dshift=FAKE, dw=None, dwp=None, ws=FAKE, wsb=0):
    return rc.lib().rc_gated_norm_backward(ctypes.byref(d), dy, lddy, dh, lddh, h, ldh, x, ldx, gate, scale, w, wp, dhi,
                                           lddhi, dx, lddx, dgate, dscale, dshift, dw, dwp, ws, wsb, None)


@pytest.mark.parametrize("bad,status", [
    (dict(h=None), "ARG"), (dict(dy=FAKE + 2), "ARG"), (dict(lddy=32), "ARG"), (dict(lddh=65), "ARG"), (dict(dhi=None), "ARG"),
    (dict(dx=None), "ARG"), (dict(x=None), "ARG"), (dict(x=None, dx=None), "ARG"), (dict(dy=None), "ARG"),
    (dict(dy=None, dh=None, scale=None, dscale=None, dshift=None), "ARG"), (dict(dw=FAKE), "ARG"), (dict(dwp=FAKE), "ARG"),
    (dict(gate=None), "ARG"), (dict(wp=FAKE), "ARG"), (dict(dgate=FAKE + 2), "ARG"), (dict(lddhi=128), "ARG"), (dict(lddx=128), "ARG"),
    (dict(), "WORKSPACE"), (dict(ws=None, wsb=1 << 40), "WORKSPACE"), (dict(ws=FAKE + 8, wsb=1 << 40), "WORKSPACE")],
    ids=lambda x: "-".join(f"{k}" for k in x) if isinstance(x, dict) else x)
def test_norm_gradient_refusals(bad, status):
    assert norm_bwd(desc(), **bad) == getattr(rc, "RC_ERR_" + status), message()


def test_norm_gradient_of_too_many_vectors():
    d = desc(B=2, G=32768)
    assert norm_bwd(d, wsb=1 << 40) == rc.RC_ERR_UNSUPPORTED and "65536" in message()
    d = desc(B=65535, G=65535)
    assert norm_bwd(d, wsb=1 << 40) == rc.RC_ERR_UNSUPPORTED
    assert norm_bwd(desc(B=2, G=32767), wsb=0) == rc.RC_ERR_WORKSPACE


def test_norm_chunks_of_many_entries_are_found_at_once():
    """More entries and spans than CUs: one chunk per span, without a search over every row count."""
    t0 = time.perf_counter()
    for B, spans in ((512, ((4000, 0),)), (60_000, ((1, 0), (30_000, 1))), (9, ((1, 0),) * 31 + ((200_000_000, 1),)),
                     (129, ((1, 0), (8_000_000, 1)))):
        d = desc(B=B, C=64, N=sum(n for n, _ in spans), spans=spans)
        need = rc.lib().rc_gated_norm_backward_workspace_bytes(ctypes.byref(d))
        assert need == B * len(spans) * 3 * 64 * 4
    assert time.perf_counter() - t0 < 0.5


def test_norm_workspace_is_one_round_of_chunks():
    """Three sums of C floats per chunk; no more chunks than CUs, whatever the spans."""
    for spans in (((4096, 0),), ((37, 1), (203, 0), (1577, 0), (1600, 1), (519, 1)), ((1, 0),) * 32, ((9, 0), (100_000, 1))):
        for B in (1, 2, 3):
            N = sum(n for n, _ in spans)
            d = desc(B=B, C=128, N=N, spans=spans)
            chunks = rc.lib().rc_gated_norm_backward_workspace_bytes(ctypes.byref(d)) / (3 * 128 * 4)
            assert chunks == int(chunks) and len(spans) * B <= chunks <= max(256, len(spans) * B)


def test_launches_beyond_32_bits_of_threads():
    """Refused before any HIP call (the calls that fit fail later, at their workspace, or are not made)."""
    L = rc.Layout([(1, 4), (2, 4)], "dense")
    assert bwd(L, B=65535, H=65535, D=64) == rc.RC_ERR_ARG and "grid limit" in message()
    assert bwd(L, B=4096, H=2047, D=64) == rc.RC_ERR_WORKSPACE
    R = init()[1]
    assert rot(R, B=1, N=(1 << 26) + 1, H=1) == rc.RC_ERR_ARG and "grid limit" in message()
    assert rot_bwd(R, B=2, N=(1 << 26), H=1) == rc.RC_ERR_ARG and "grid limit" in message()
    n = 1 << 24
    assert norm(desc(B=4, N=n, spans=((n, 0),))) == rc.RC_ERR_ARG and "grid limit" in message()
    assert norm(desc(B=1, C=2048, N=n, mb=0, mg=0, spans=((n, 0),)), ldh=2048, ldx=2048, ldho=2048, ldy=2048) == rc.RC_ERR_ARG
    assert "grid limit" in message()


# ---------------------------------------------------------------- binding
def test_binding_takes_gpu_tensors_only():
    L = rc.Layout(SEGS, "perref")
    q = torch.zeros(1, 152, 2, 64, dtype=torch.bfloat16)
    lse = torch.zeros(1, 2, 152)
    with pytest.raises(ValueError, match="GPU tensor"):
        rc.full_attention_backward(L, q, q, q, q, lse, q)
    R = rc.Rotary(64, (16, 24, 24))
    pos = torch.zeros(152, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensor"):
        rc.qk_rotary(R, q, q, pos)
    with pytest.raises(ValueError, match="GPU tensor"):
        rc.qk_rotary_backward(R, q, None, pos)
    with pytest.raises(ValueError, match="q, k or both"):
        rc.qk_rotary(R, None, None, pos)
    h = torch.zeros(1, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU tensor"):
        rc.gated_norm(h)
    with pytest.raises(ValueError, match="GPU tensor"):
        rc.gated_norm_backward(h, h)


def test_modulation_spans():
    L = rc.Layout(SEGS, "perref")
    assert L.modulation_spans() == [(8, 1), (16, 0), (64, 0), (64, 1)]
    assert L.modulation_spans(rc.ROWS_LIVE, live=3) == [(16, 3), (64, 3)]
    assert L.modulation_spans(rc.ROWS_STATIC, static=0) == [(8, 0), (64, 0)]
