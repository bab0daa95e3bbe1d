"""Planner cases of the layer operators for the sanitizer build (run by
test_host_sanitized_layer.py; skipped otherwise).  Pointers are fake."""
import ctypes
import os
import random

import pytest

import paper_2608_21229_amd as rc
from tests.test_capi_host import random_layout
from tests.test_layer_capi import FAKE, bwd, desc, init, norm, norm_bwd, rot, rot_bwd

pytestmark = pytest.mark.skipif(not os.environ.get("REFCACHE_STUB"), reason="needs the stub-launcher build")


def stub(name, *args):
    f = getattr(rc.lib(), "rc_stub_layer_" + name)
    f.restype = ctypes.c_long
    return f(*args)


@pytest.mark.parametrize("preset", ["paper", "perref", "isolated", "dense", "random"])
def test_random_layouts(preset):
    rng = random.Random(17)
    split = 0
    for _ in range(200):
        kinds, lens = random_layout(rng)
        n = len(kinds)
        mask = [[rng.random() < 0.5 for _ in range(n)] for _ in range(n)] if preset == "random" else preset
        L = rc.Layout(list(zip(kinds, lens)), mask)
        B, H, D = rng.choice([1, 2]), rng.choice([1, 2, 5, 24, 64]), rng.choice([64, 128])
        need = L.backward_workspace_bytes(B, H, D)
        n0 = stub("launches")
        assert bwd(L, B=B, H=H, D=D, ws=FAKE, wsb=need - 1) == rc.RC_ERR_WORKSPACE
        assert bwd(L, B=B, H=H, D=D, ws=FAKE, wsb=need) == rc.RC_OK
        assert stub("launches") == n0 + 1
        assert stub("pairs", 0) == L.pairs(rc.ENTRY_FULL) == stub("pairs", 1)
        rows = 2 * ((B * H * sum(lens) * 4 + 15) // 16 * 16)
        assert need == rows + B * H * stub("slots") * stub("own") * D * 4
        split += stub("slots") > 0 or stub("own") == 128
    assert split > 20, "few layouts of the draw are split or have small own tiles"


@pytest.mark.parametrize("D", [64, 128])
def test_own_tiles(D):
    """Large ones where heads fill the chip, small ones for few rows or heads (test_gpu_backward.py relies on both)."""
    layouts = [([(2, n)], "dense") for n in (129, 160, 191, 193, 224, 255, 256, 257, 320, 513)]
    layouts += [([(0, 257), (1, 33), (2, 300), (3, 255), (3, 1)], p) for p in ("perref", "paper", "isolated", "dense")]
    for segs, preset in layouts:
        L = rc.Layout(segs, preset)
        assert bwd(L, B=2, H=128, D=D, wsb=1 << 40) == rc.RC_OK and stub("own") == 256, (segs, preset)
        assert bwd(L, B=1, H=2, D=D, wsb=1 << 40) == rc.RC_OK and stub("own") == 128, (segs, preset)


def test_largest_table():
    L = rc.Layout([(2, 300)] * 32, "dense")
    assert bwd(L, wsb=1 << 40) == rc.RC_OK
    assert stub("pairs", 0) == (300 * 32) ** 2


def test_rotation_and_norm_calls():
    R = init()[1]
    for N, H in ((1, 1), (5, 3), (4096, 24), (100_000, 1)):
        for q, k in ((FAKE, FAKE), (FAKE, None), (None, FAKE)):
            assert rot(R, N=N, H=H, q=q, k=k, ts=H * 128, os_=H * 128) == rc.RC_OK
            assert rot_bwd(R, N=N, H=H, dq=q, dk=k, gs=H * 128, os_=H * 128) == rc.RC_OK
            need = rc.lib().rc_rotary_backward_workspace_bytes(ctypes.byref(R), 1, N)
            assert rot_bwd(R, N=N, H=H, dq=q, dk=k, gs=H * 128, ts=H * 128, os_=H * 128, qn=q, kn=k, ws=FAKE, wsb=need) == rc.RC_OK
    rng = random.Random(3)
    for _ in range(300):
        spans = [(rng.choice([0, 1, 7, 64, 1000, 5000]), rng.randint(0, 3)) for _ in range(rng.randint(1, 32))]
        B = rng.choice([1, 2, 7])
        d = desc(B=B, G=4, N=sum(n for n, _ in spans), spans=spans)
        assert norm(d) == rc.RC_OK
        need = rc.lib().rc_gated_norm_backward_workspace_bytes(ctypes.byref(d))
        assert norm_bwd(d, wsb=need) == rc.RC_OK
        assert need == B * stub("chunks") * 3 * 64 * 4
