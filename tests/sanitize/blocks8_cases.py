"""Planner cases of the 8-bit projections for the sanitizer build (run by
test_host_sanitized_blocks8.py; skipped otherwise).  Pointers are fake."""
import ctypes
import os
import random

import pytest

import paper_2608_21229_amd as rc
from tests.test_blocks8_capi import FAKE, back, dequant, linear, linear_blocks, quant

pytestmark = pytest.mark.skipif(not os.environ.get("REFCACHE_STUB"), reason="needs the stub-launcher build")
WS = FAKE + (1 << 36)


def stub(name, *args):
    f = getattr(rc.lib(), "rc_stub_blocks8_" + name)
    f.restype = ctypes.c_long
    f.argtypes = [ctypes.c_size_t, ctypes.c_long][:len(args)]
    return f(*args)


def sizes(rng):
    n = lambda: 8 * int(round(2 ** rng.uniform(0, 10)))  # noqa: E731
    return int(round(2 ** rng.uniform(0, 18))), n(), n()


def test_random_calls():
    rng = random.Random(5)
    seen, few, split, whole = set(), 0, 0, 0
    for _ in range(400):
        M, N, K = sizes(rng)
        stub("workspace", 0, 0)
        n0 = stub("launches")
        assert quant(M=N, K=K, ldx=K, out_t=None) == quant(M=N, K=K, ldx=K) == quant(M=M, K=K, ldx=K, square=0, out_t=None) == 0
        assert dequant(M=M, K=K, ldo=K) == linear_blocks(M=M, N=N, K=K, ldo=N) == rc.RC_OK
        assert stub("launches") == n0 + 5
        seen.add(stub("tile"))
        need = rc.lib().rc_linear_fp8_workspace_bytes(M, N, K)
        stub("workspace", WS, need)
        if need:
            assert linear(M=M, N=N, K=K, lda=K, ldo=N, ws=WS, wsb=need - 1) == rc.RC_ERR_WORKSPACE
        n0 = stub("launches")
        assert linear(M=M, N=N, K=K, lda=K, ldo=N, ws=WS, wsb=need) == rc.RC_OK
        assert stub("launches") == n0 + (2 if need else 1) and stub("few") == (need == 0)
        few += need == 0
        need = rc.lib().rc_linear_fp8_backward_workspace_bytes(M, N, K, 1, 1)
        stub("workspace", WS, need)
        if need:
            assert back(M=M, N=N, K=K, lddy=N, lddx=K, lddw=K, ws=WS, wsb=need - 1) == rc.RC_ERR_WORKSPACE
        assert back(M=M, N=N, K=K, lddy=N, lddx=K, lddw=K, ws=WS, wsb=need) == rc.RC_OK
        split += stub("splits") > 1
        whole += stub("whole") > 0
        need = rc.lib().rc_linear_fp8_backward_workspace_bytes(M, N, K, 0, 1)
        stub("workspace", WS, need)
        assert back(M=M, N=N, K=K, lddy=N, dx=None, w_t=None, lddw=K, ws=WS, wsb=need) == rc.RC_OK
    assert seen == {0, 1, 2, 3, 4, 5} and few > 40 and split > 100 and whole > 2


def test_limits_of_the_grid():
    """The largest sizes plan without an overflow, or are refused."""
    for M, N, K in ((1 << 28, 8, 8), (1 << 28, 1 << 22, 1 << 22), (1, 1 << 22, 1 << 22), (1 << 20, 1 << 22, 8), (1 << 28, 8, 1 << 22),
                    (17, 1 << 22, 1 << 22)):
        stub("workspace", 0, 0)
        ld = dict(M=M, N=N, K=K)
        assert linear(lda=K, ldo=N, wsb=1 << 62, **ld) in (rc.RC_OK, rc.RC_ERR_ARG)
        assert linear_blocks(ldo=N, **ld) in (rc.RC_OK, rc.RC_ERR_ARG)
        assert back(lddy=N, lddx=K, lddw=K, wsb=1 << 62, **ld) in (rc.RC_OK, rc.RC_ERR_ARG)
    stub("workspace", 0, 0)
    assert back(M=0, N=1 << 18, K=1 << 18, lddw=1 << 18, dx=None, x=None, w_t=None) == rc.RC_OK
    assert back(M=0, N=1 << 22, K=1 << 22, lddw=1 << 22, dx=None, x=None, w_t=None) == rc.RC_ERR_ARG
