"""Host-only checks of the 8-bit projections: what the C ABI and the binding
refuse, with which status, before any HIP call; workspaces.  Pointers are fake and
never dereferenced: every call below fails validation or has nothing to do."""
import ctypes

import pytest
import torch

import paper_2608_21229_amd as rc
from paper_2608_21229_amd import binding

FAKE = 0x7f0000000000
ids = lambda x: "-".join(x) if isinstance(x, dict) else x  # noqa: E731


def message():
    return rc.lib().rc_last_error().decode()


def blocks(rows, cols, codes=FAKE, ld=None, exps=FAKE, le=None):
    return binding.rc_blocks8(codes, -(-cols // 128) * 128 if ld is None else ld, exps,
                              -(-rows // 16) * 16 if le is None else le)


def ref(b):
    return None if b is None else ctypes.byref(b)


def quant(M=40, K=136, x=FAKE, ldx=136, square=1, out=Ellipsis, out_t=Ellipsis):
    out = blocks(M, K) if out is Ellipsis else out
    out_t = blocks(K, M) if out_t is Ellipsis else out_t
    return rc.lib().rc_quantize_blocks(M, K, x, ldx, square, ref(out), ref(out_t), None)


SIZES = [(dict(M=-1), "ARG"), (dict(M=(1 << 28) + 1), "ARG"), (dict(K=0), "ARG"), (dict(K=-8), "ARG"), (dict(K=132), "UNSUPPORTED"),
         (dict(K=(1 << 22) + 8), "UNSUPPORTED")]


@pytest.mark.parametrize("bad,status", SIZES + [
    (dict(x=None), "ARG"), (dict(x=FAKE + 8), "ARG"), (dict(ldx=128), "ARG"), (dict(ldx=140), "ARG"),
    (dict(ldx=(1 << 22) + 8), "ARG"), (dict(out=None), "ARG"), (dict(out=blocks(40, 136, codes=None)), "ARG"),
    (dict(out=blocks(40, 136, codes=FAKE + 4)), "ARG"), (dict(out=blocks(40, 136, exps=None)), "ARG"),
    (dict(out=blocks(40, 136, exps=FAKE + 1)), "ARG"), (dict(out=blocks(40, 136, ld=128)), "ARG"),
    (dict(out=blocks(40, 136, ld=264)), "ARG"), (dict(out=blocks(40, 136, le=32)), "ARG"),
    (dict(out=blocks(40, 136, le=56)), "ARG"), (dict(out=blocks(40, 136, le=(1 << 28) + 16)), "ARG"),
    (dict(out=blocks(40, 136, ld=(1 << 22) + 16)), "ARG"), (dict(out_t=blocks(136, 40, ld=64)), "ARG"),
    (dict(out_t=blocks(136, 40, le=128)), "ARG"), (dict(square=0), "UNSUPPORTED"),
    (dict(M=44, out_t=blocks(136, 44)), "UNSUPPORTED")], ids=ids)
def test_quantize_refusals(bad, status):
    assert quant(**bad) == getattr(rc, "RC_ERR_" + status), message()
    assert message()


def dequant(M=40, K=136, x=Ellipsis, out=FAKE, ldo=136):
    x = blocks(M, K) if x is Ellipsis else x
    return rc.lib().rc_dequantize_blocks(M, K, ref(x), out, ldo, None)


@pytest.mark.parametrize("bad,status", SIZES + [
    (dict(x=None), "ARG"), (dict(x=blocks(40, 136, ld=128)), "ARG"), (dict(out=None), "ARG"), (dict(out=FAKE + 2), "ARG"),
    (dict(ldo=128), "ARG"), (dict(ldo=137), "ARG")], ids=ids)
def test_dequantize_refusals(bad, status):
    assert dequant(**bad) == getattr(rc, "RC_ERR_" + status), message()


def linear(M=100, N=72, K=136, a=FAKE, lda=136, w=Ellipsis, r=None, ldr=0, out=FAKE, ldo=72, ws=FAKE, wsb=1 << 40):
    w = blocks(N, K) if w is Ellipsis else w
    return rc.lib().rc_linear_fp8(M, N, K, a, lda, ref(w), r, ldr, out, ldo, ws, wsb, None)


def linear_blocks(M=100, N=72, K=136, a=Ellipsis, w=Ellipsis, r=None, ldr=0, out=FAKE, ldo=72):
    a, w = blocks(M, K) if a is Ellipsis else a, blocks(N, K) if w is Ellipsis else w
    return rc.lib().rc_linear_fp8_blocks(M, N, K, ref(a), ref(w), r, ldr, out, ldo, None)


PRODUCT = SIZES + [(dict(N=0), "ARG"), (dict(N=68), "UNSUPPORTED"), (dict(N=(1 << 22) + 8), "UNSUPPORTED"),
                   (dict(w=None), "ARG"), (dict(w=blocks(72, 136, ld=128)), "ARG"), (dict(w=blocks(72, 136, le=64)), "ARG"),
                   (dict(out=None), "ARG"), (dict(out=FAKE + 4), "ARG"), (dict(ldo=64), "ARG"), (dict(ldo=76), "ARG"),
                   (dict(r=FAKE + 8, ldr=72), "ARG"), (dict(r=FAKE, ldr=64), "ARG"), (dict(r=FAKE, ldr=1 << 23), "ARG")]


@pytest.mark.parametrize("bad,status", PRODUCT + [(dict(a=None), "ARG"), (dict(a=blocks(100, 136, ld=128)), "ARG"),
                                                  (dict(a=blocks(100, 136, le=96)), "ARG")], ids=ids)
def test_product_of_blocks_refusals(bad, status):
    assert linear_blocks(**bad) == getattr(rc, "RC_ERR_" + status), message()


BIG = dict(M=1000, N=4096, K=4096, lda=4096, ldo=4096)


@pytest.mark.parametrize("bad,status", PRODUCT + [
    (dict(a=None), "ARG"), (dict(a=FAKE + 2), "ARG"), (dict(lda=128), "ARG"), (dict(lda=139), "ARG"),
    (dict(BIG, ws=None), "WORKSPACE"), (dict(BIG, ws=FAKE + 8), "WORKSPACE"), (dict(BIG, wsb=1000 * 4096), "WORKSPACE")], ids=ids)
def test_product_refusals(bad, status):
    assert linear(**bad) == getattr(rc, "RC_ERR_" + status), message()


def test_product_workspace():
    need = rc.lib().rc_linear_fp8_workspace_bytes
    assert need(1000, 4096, 4096) == 1000 * 4096 + 32 * 1008
    assert need(1000, 4096, 4104) == 1000 * 4224 + 33 * 1008
    assert need(32, 1 << 20, 1 << 20) == 0 and need(80, 384, 128) == 0 and need(0, 8, 8) == 0
    assert need(33, 7680, 2560) > 0
    assert need(-1, 8, 8) == need(8, 9, 8) == need(8, 8, 0) == 0


def back(M=100, N=72, K=136, dy=FAKE, lddy=72, x=Ellipsis, w_t=Ellipsis, r=None, ldr=0, dx=FAKE, lddx=136, dw=FAKE, lddw=136,
         ws=FAKE, wsb=1 << 40):
    x, w_t = blocks(M, K) if x is Ellipsis else x, blocks(K, N) if w_t is Ellipsis else w_t
    return rc.lib().rc_linear_fp8_backward(M, N, K, dy, lddy, ref(x), ref(w_t), r, ldr, dx, lddx, dw, lddw, ws, wsb, None)


@pytest.mark.parametrize("bad,status", SIZES + [
    (dict(N=0), "ARG"), (dict(N=68), "UNSUPPORTED"), (dict(dy=None), "ARG"), (dict(dy=FAKE + 8), "ARG"), (dict(lddy=64), "ARG"),
    (dict(dx=None, dw=None, x=None, w_t=None), "ARG"), (dict(dx=None), "ARG"), (dict(dx=None, w_t=None, r=FAKE, ldr=136), "ARG"),
    (dict(dw=None), "ARG"), (dict(x=None), "ARG"), (dict(w_t=None), "ARG"), (dict(w_t=blocks(72, 136)), "ARG"),
    (dict(x=blocks(64, 136)), "ARG"), (dict(dx=FAKE + 2), "ARG"), (dict(lddx=128), "ARG"), (dict(r=FAKE + 2, ldr=136), "ARG"),
    (dict(r=FAKE, ldr=128), "ARG"), (dict(dw=FAKE + 4), "ARG"), (dict(lddw=132), "ARG"), (dict(lddw=1 << 23), "ARG"),
    (dict(M=20000, N=1024, K=1024, lddy=1024, lddx=1024, lddw=1024, wsb=20000 * 1024), "WORKSPACE"),
    (dict(M=20000, N=1024, K=1024, lddy=1024, lddx=1024, lddw=1024, ws=None), "WORKSPACE")], ids=ids)
def test_gradient_refusals(bad, status):
    assert back(**bad) == getattr(rc, "RC_ERR_" + status), message()


def test_gradient_workspace():
    need = rc.lib().rc_linear_fp8_backward_workspace_bytes
    both, dx, dw = (need(20000, 1024, 2048, *w) for w in ((1, 1), (1, 0), (0, 1)))
    assert dx == 20000 * 1024 + 8 * 20000 and both == dx + dw and dw % (1024 * 2048 * 4) == 0 and dw > 0
    assert need(80, 384, 128, 1, 1) == 0 == need(100, 9, 8, 1, 1) == need(-1, 8, 8, 1, 1)


def test_no_rows_and_launch_limits():
    assert quant(M=0, x=None, out=None, out_t=None) == rc.RC_OK
    assert dequant(M=0, x=None, out=None) == rc.RC_OK
    assert linear(M=0, a=None, out=None, ws=None, wsb=0) == linear_blocks(M=0, a=None, out=None) == rc.RC_OK
    assert back(M=0, dx=None, dw=None, dy=None, x=None, w_t=None, ws=None, wsb=0) == rc.RC_OK
    # a launch has fewer than 2^32 threads: refused by the call, and 0 from the queries
    big = dict(M=1 << 28, N=1 << 22, K=128)
    assert linear(lda=128, ldo=1 << 22, **big) == rc.RC_ERR_ARG and "launch" in message()
    assert linear_blocks(ldo=1 << 22, **big) == rc.RC_ERR_ARG and "launch" in message()
    assert rc.lib().rc_linear_fp8_workspace_bytes(*big.values()) == 0
    assert back(lddy=1 << 22, lddx=128, lddw=128, **big) == rc.RC_ERR_ARG and "launch" in message()
    assert quant(M=1 << 28, K=1 << 22, ldx=1 << 22, square=0, out_t=None) == rc.RC_ERR_ARG and "launch" in message()
    assert dequant(M=1 << 28, K=1 << 20, ldo=1 << 20) == rc.RC_ERR_ARG and "launch" in message()
    assert rc.lib().rc_linear_fp8_backward_workspace_bytes(1 << 28, 1 << 22, 128, 1, 0) == 0


# ---------------------------------------------------------------- the binding
def cpu_blocks(rows, cols, t=None):
    return rc.Fp8Blocks(torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.uint8),
                        torch.zeros(-(-cols // 128), -(-rows // 16) * 16, dtype=torch.uint8), (rows, cols), t)


def test_binding_refuses_host_tensors_and_other_types():
    x, b = torch.zeros(4, 128, dtype=torch.bfloat16), cpu_blocks(4, 128)
    for call in (lambda: rc.quantize_blocks(x), lambda: rc.dequantize_blocks(b), lambda: rc.linear_fp8(x, b),
                 lambda: rc.linear_fp8(b, b), lambda: rc.linear_fp8_backward(x, b, b), lambda: rc.dequantize_blocks(x),
                 lambda: rc.quantize_blocks(x.float()), lambda: rc.linear_fp8(b, x)):
        with pytest.raises(ValueError, match="GPU|Fp8Blocks"):
            call()


def test_blocks_shapes():
    assert cpu_blocks(5, 136).shape == (5, 136)
    with pytest.raises(ValueError, match="codes must be"):
        rc.Fp8Blocks(torch.zeros(5, 136, dtype=torch.uint8), torch.zeros(2, 16, dtype=torch.uint8), (5, 136))
    with pytest.raises(ValueError, match="exps must be"):
        rc.Fp8Blocks(torch.zeros(5, 256, dtype=torch.uint8), torch.zeros(2, 5, dtype=torch.uint8), (5, 136))
    with pytest.raises(ValueError, match="uint8"):
        rc.Fp8Blocks(torch.zeros(5, 256, dtype=torch.int8), torch.zeros(2, 16, dtype=torch.uint8), (5, 136))
    with pytest.raises(ValueError, match="t must be"):
        cpu_blocks(8, 136, cpu_blocks(8, 136))
    assert cpu_blocks(8, 136, cpu_blocks(136, 8)).t.shape == (136, 8)


def test_strided_workspaces_are_refused():
    """A workspace is written as one run of bytes: a view of every second has half of them."""
    dev, whole = torch.device("cpu"), torch.zeros(128, dtype=torch.uint8)
    assert binding._workspace(whole, 64, dev, None) is whole
    with pytest.raises(ValueError, match="contiguous"):
        binding._workspace(whole[::2], 64, dev, None)
    with pytest.raises(ValueError, match="contiguous"):
        binding._workspace(torch.zeros(16, 8, dtype=torch.float32)[:, :4], 64, dev, None)
    with pytest.raises(ValueError, match="contiguous"):
        binding._workspace(torch.zeros(1, dtype=torch.uint8).expand(64), 64, dev, None)


def test_outputs_over_inputs_are_refused():
    """Tiles are written while others still read: an output may be the residual as it lies, and nothing else."""
    m = torch.zeros(8, 512, dtype=torch.bfloat16)
    x, other = m[:, :128], m[:, 128:256]
    binding._apart(x, "out", 512, other, "a", x, 512)
    binding._apart(x, "out", 512, other, "a", None, 0)
    binding._apart(m[:0], "out", 512, m[:0], "a", None, 0)
    with pytest.raises(ValueError, match="out may not be a"):
        binding._apart(x, "out", 512, x, "a", None, 0)
    with pytest.raises(ValueError, match="stride"):
        binding._apart(x, "out", 512, other, "a", m.view(32, 128)[:8], 128)
