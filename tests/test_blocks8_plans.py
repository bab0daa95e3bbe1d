"""The sizes at which the weights' gradient is tested on the GPU take the plans that
they are there for: the host code with the stub launchers, CPU only."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_21229_amd import binding
from tests.blocks8_plans import TILES, WEIGHT_GRADIENTS, workspace_bytes
from tests.test_blocks8_capi import FAKE, blocks
from tests.test_host_sanitized import CSRC, ROOT


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("host") / "librefcache_host.so")
    san = os.path.join(ROOT, "tests", "sanitize")
    build = ["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
             os.path.join(CSRC, "layout.cpp"), os.path.join(CSRC, "api.cpp"), os.path.join(san, "stub_launchers.cpp"),
             os.path.join(san, "stub_blocks8.cpp"), "-o", path]
    r = subprocess.run(build, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = ctypes.CDLL(path)
    for name in ("rc_linear_fp8_backward", "rc_linear_fp8_backward_workspace_bytes"):
        f = getattr(lib, name)
        f.restype, f.argtypes = binding.SIGNATURES[name]
    for name in ("tile", "splits", "whole"):
        getattr(lib, "rc_stub_blocks8_" + name).restype = ctypes.c_long
    return lib


@pytest.mark.parametrize("plan", WEIGHT_GRADIENTS, ids=str)
def test_weight_gradient_plans(host, plan):
    m, n, k, tile, shares, whole, tiles = plan
    bm, bn = TILES[tile]
    assert tiles == -(-n // bm) * -(-k // bn) and (shares == 1 or tiles > whole)
    need = host.rc_linear_fp8_backward_workspace_bytes(m, n, k, 0, 1)
    assert need == workspace_bytes(plan)
    x = blocks(m, k)
    assert host.rc_linear_fp8_backward(m, n, k, FAKE, n, ctypes.byref(x), None, None, 0, None, 0, FAKE, k, FAKE, need, None) == 0
    assert (host.rc_stub_blocks8_tile(), host.rc_stub_blocks8_splits(), host.rc_stub_blocks8_whole()) == (tile, shares, whole)


@pytest.mark.parametrize("plan", [p for p in WEIGHT_GRADIENTS if p[4] > 1], ids=str)
def test_workspaces_tell_the_plans_with_shares(plan):
    """No other tile or number of shares needs as many bytes, so the size alone shows the plan."""
    _, n, k, tile, shares, _, _ = plan
    for t, (bm, bn) in enumerate(TILES):
        rest = -(-n // bm) * -(-k // bn) % 256
        for j in range(2, 256 // rest + 1 if rest else 0):
            assert (rest * j * bm * bn * 4 == workspace_bytes(plan)) == ((t, j) == (tile, shares))
