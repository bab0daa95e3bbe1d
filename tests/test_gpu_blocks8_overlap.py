"""The 8-bit projections' entry points with outputs and workspaces in their inputs'
buffers: refused where they share memory, before anything is launched; exact beside them."""
import pytest
import torch

import paper_2608_21229_amd as rc
from tests import blocks8_plain as plain
from tests.test_blocks8_overlap import blocks_of

pytestmark = pytest.mark.gpu

M, N, K = 70, 264, 264  # one shape for a, out, dy and dx


def gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.fixture(scope="module")
def weights():
    return rc.quantize_blocks(plain.rows(gen(1), N, K), square=True, transposed=True)


@pytest.mark.parametrize("rows,cols", [(1, 0), (0, 8), (3, 16)])
@pytest.mark.parametrize("few", [False, True])
def test_shifted_outputs_are_refused(weights, rows, cols, few):
    m = 9 if few else M
    buf = plain.rows(gen(2), M + 8, 512)
    keep = buf.clone()
    x, over, other = buf[:m, :K], buf[rows:m + rows, cols:K + cols], plain.rows(gen(3), m, K)
    x8 = rc.quantize_blocks(other)
    with pytest.raises(ValueError, match="out may not be a"):
        rc.linear_fp8(x, weights, out=over)
    for a in (other, x8):
        with pytest.raises(ValueError, match="residual as it lies"):
            rc.linear_fp8(a, weights, residual=x, out=over)
    with pytest.raises(ValueError, match="dx may not be dy"):
        rc.linear_fp8_backward(x, x8, weights, dx=over)
    with pytest.raises(ValueError, match="residual as it lies"):
        rc.linear_fp8_backward(other, x8, weights, residual=x, dx=over)
    assert torch.equal(buf, keep)


def test_outputs_over_codes_are_refused(weights):
    dy, pool = plain.rows(gen(4), M, N), torch.zeros(1 << 18, dtype=torch.uint8, device="cuda")
    x8 = blocks_of(pool, 0, M, K)
    over = pool[16:16 + M * K * 2].view(torch.bfloat16).view(M, K)
    for what, call in (("x", lambda: rc.quantize_blocks(over, out=x8)), ("x", lambda: rc.dequantize_blocks(x8, out=over)),
                       ("a", lambda: rc.linear_fp8(x8, weights, out=over)),
                       ("x", lambda: rc.linear_fp8_backward(dy, x8, weights, dx=over)),
                       ("w", lambda: rc.linear_fp8(dy, blocks_of(pool, 16, N, K), out=over))):
        with pytest.raises(ValueError, match="out|dx") as e:
            call()
        assert f"may not overlap {what}" in str(e.value)
    dw = torch.empty(N, K, device="cuda")
    with pytest.raises(ValueError, match="dw may not overlap dx"):
        rc.linear_fp8_backward(dy, x8, weights, dw=dw, dx=dw.view(-1)[:M * K // 2].view(torch.bfloat16).view(M, K))
    assert not pool.any()


def test_workspaces_over_inputs_and_outputs_are_refused(weights):
    m = 1400
    assert rc.lib().rc_linear_fp8_workspace_bytes(m, N, K) > 0
    x, r, out = (plain.rows(gen(i), m, K) for i in (5, 6, 7))
    x8 = rc.quantize_blocks(x)
    keep = [t.clone() for t in (x, r, out)]
    for what, ws in (("a", x), ("residual", r), ("out", out)):
        with pytest.raises(ValueError, match=f"workspace may not overlap {what}"):
            rc.linear_fp8(x, weights, residual=r, out=out, workspace=ws)
    for what, ws in (("dy", x), ("residual", r), ("dx", out)):
        with pytest.raises(ValueError, match=f"workspace may not overlap {what}"):
            rc.linear_fp8_backward(x, x8, weights, residual=r, dx=out, want_dw=False, workspace=ws)
    pool = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    assert 16 < rc.lib().rc_linear_fp8_backward_workspace_bytes(m, N, K, 1, 1) <= pool.numel()
    with pytest.raises(ValueError, match="workspace may not overlap x"):
        rc.linear_fp8_backward(x, blocks_of(pool, 16, m, K), weights, workspace=pool)
    assert all(torch.equal(a, b) for a, b in zip((x, r, out), keep))


@pytest.mark.parametrize("m", [9, 70, 1400])
def test_side_by_side_in_one_buffer(weights, m):
    """Input, residual and output as columns of one buffer, and a workspace behind the output's last byte."""
    buf = plain.rows(gen(8), m, 1024)
    x, r, out = buf[:, :K], buf[:, 264:528], buf[:, 528:792]
    keep, x8 = buf.clone(), rc.quantize_blocks(x)
    want = [rc.linear_fp8(x, weights, residual=r), rc.linear_fp8(x8, weights, residual=r),
            rc.linear_fp8_backward(x, x8, weights, residual=r)[0]]
    pool = torch.zeros(1 << 21, dtype=torch.uint8, device="cuda")
    for i, call in enumerate((lambda: rc.linear_fp8(x, weights, residual=r, out=out, workspace=pool),
                              lambda: rc.linear_fp8(x8, weights, residual=r, out=out),
                              lambda: rc.linear_fp8_backward(x, x8, weights, residual=r, dx=out, workspace=pool)[0])):
        assert call() is out and torch.equal(out, want[i])
        assert torch.equal(buf[:, :528], keep[:, :528]) and torch.equal(buf[:, 792:], keep[:, 792:])
    need = rc.lib().rc_linear_fp8_workspace_bytes(m, N, K)
    at = -(-need // 16) * 16
    behind = pool[at:at + m * N * 2].view(torch.bfloat16).view(m, N)
    assert torch.equal(rc.linear_fp8(x, weights, residual=r, out=behind, workspace=pool), want[0])
