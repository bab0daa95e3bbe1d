"""The 8-bit projections beyond 32-bit offsets: rows far apart in wide buffers, and
codes of more than 4 GiB.  Rows are independent of each other, so a window's bits are
those of a call of the window alone."""
import pytest
import torch

import paper_2608_21229_amd as rc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=BF16)


def test_rows_far_apart():
    m, n, k, ld = 1100, 136, 264, 1 << 21  # 4.6 GB from the first row to the last
    g = gen(1)
    x, w8 = randn(g, m, k), rc.quantize_blocks(randn(g, n, k), square=True, transposed=True)
    dy, r = randn(g, m, n), randn(g, m, k)

    def wide(t):
        v = torch.empty(m * ld, dtype=BF16, device="cuda").as_strided((m, t.shape[1]), (ld, 1))
        v.copy_(t)
        return v

    x8 = rc.quantize_blocks(x)
    far = wide(x)
    got = rc.quantize_blocks(far)
    assert torch.equal(got.codes, x8.codes) and torch.equal(got.exps[:, :m], x8.exps[:, :m])
    assert torch.equal(rc.dequantize_blocks(x8, out=far), rc.dequantize_blocks(x8))
    want = rc.quantize_blocks(x[:1096], square=True, transposed=True)
    got = rc.quantize_blocks(wide(x)[:1096], square=True, transposed=True)
    assert torch.equal(got.codes, want.codes) and torch.equal(got.t.codes, want.t.codes)
    out = rc.linear_fp8(x8, w8)
    assert torch.equal(rc.linear_fp8(x8, w8, out=wide(dy)), out)
    few = rc.linear_fp8(x[:30], w8)
    far = wide(x)
    assert torch.equal(rc.linear_fp8(far[:30], w8), few)
    assert torch.equal(rc.linear_fp8(far[-30:], w8), rc.linear_fp8(x[-30:], w8))
    dx, dw = rc.linear_fp8_backward(dy, x8, w8, residual=r)
    del far
    far = wide(dy)
    got_dx, got_dw = rc.linear_fp8_backward(far, x8, w8, residual=r)
    assert torch.equal(got_dx, dx) and torch.equal(got_dw, dw)


def test_codes_beyond_4_gib():
    m, n, k = 1 << 20, 136, 4104  # 4.4 GB of codes
    g = gen(2)
    x = torch.empty(m, k, dtype=BF16, device="cuda").normal_(generator=g)
    w8 = rc.quantize_blocks(randn(g, n, k), square=True)
    x8 = rc.quantize_blocks(x)
    out = rc.linear_fp8(x8, w8)
    assert torch.equal(rc.linear_fp8(x, w8), out)
    back = rc.dequantize_blocks(x8)
    for at in (0, m // 2 - 7, m - 100):
        part = rc.quantize_blocks(x[at:at + 100])
        assert torch.equal(part.codes, x8.codes[at:at + 100]) and torch.equal(part.exps[:, :100], x8.exps[:, at:at + 100])
        assert torch.equal(rc.linear_fp8(part, w8), out[at:at + 100])
        assert torch.equal(rc.dequantize_blocks(part), back[at:at + 100])
    # one slice of rows that is not zero: its sums alone
    dy = torch.zeros(m, n, dtype=BF16, device="cuda")
    dy[-64:] = randn(g, 64, n)
    _, dw = rc.linear_fp8_backward(dy, x8, None, want_dx=False)
    _, want = rc.linear_fp8_backward(dy[-64:], rc.quantize_blocks(x[-64:]), None, want_dx=False)
    assert torch.equal(dw, want)


def test_two_streams_at_once():
    """Calls that overlap on one GPU share nothing."""
    g = gen(3)
    x, w8 = randn(g, 3000, 1032), rc.quantize_blocks(randn(g, 520, 1032), square=True, transposed=True)
    dy = randn(g, 3000, 520)
    x8 = rc.quantize_blocks(x)
    want = [rc.linear_fp8(x, w8), *rc.linear_fp8_backward(dy, x8, w8)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [[rc.linear_fp8(x, w8, stream=s), *rc.linear_fp8_backward(dy, x8, w8, stream=s)] for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for run in got for a, b in zip(run, want))
