"""The 8-bit products and gradients on whole numbers: their sums are exact in fp32, so
every result is known to the last bit, and one lost, doubled or misplaced value shows.

Operands are whole numbers of up to 8 (4 significant bits) times a power of two per
block, whose codes hold them exactly.  Products of the numbers and of scales up to
2^2 apart are whole multiples of the least scale below 2^8 of it: the product's cut, 2^-13 of
the largest, loses nothing, and sums of up to 2^16 of them stay whole below 2^24."""
import pytest
import torch

import paper_2608_21229_amd as rc
from tests.blocks8_plans import WEIGHT_GRADIENTS, workspace_bytes

pytestmark = pytest.mark.gpu

DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def whole(g, rows, cols, most=8):
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device=DEV).double()


def powers(g, rows, cols, base, square=False, up=1):
    """2^(base of a block column + 0 .. up of each block), [rows, cols]."""
    kb = -(-cols // 128)
    e = torch.randint(0, up + 1, (-(-rows // 128) if square else rows, kb), generator=g, device=DEV)
    if square:
        e = e.repeat_interleave(128, 0)[:rows]
    return torch.exp2((e + base).repeat_interleave(128, 1)[:, :cols].double())


def operands(seed, m, n, k):
    """a [m, k] and w [n, k] in bf16, whose blocks' powers of two take each other back, up to 2^2."""
    g = gen(seed)
    base = torch.randint(-20, 21, (1, -(-k // 128)), generator=g, device=DEV)
    a = whole(g, m, k) * powers(g, m, k, base)
    w = whole(g, n, k, 2) * powers(g, n, k, -base, square=True)
    return a, w, g


def rounded(x):
    """Whole numbers below 2^24 as a bf16 result holds them."""
    assert float(x.abs().max()) < 2 ** 24 and torch.equal(x, x.round())
    return x.float().bfloat16()


# one launch of few rows: 16 and 32 columns per work-group, 16 and 32 rows; inner lengths at which each of a
# work-group's eight waves loads its share of the blocks once, and again; last blocks of 8 to 120 values
FEW = [(1, 8, 8), (1, 2560, 1032), (2, 2560, 4616), (16, 72, 6408), (5, 4096, 8312), (2, 4104, 520), (1, 7680, 3336),
       (16, 4104, 6424), (9, 4168, 9224), (17, 520, 2056), (31, 520, 4936), (32, 40, 12296), (80, 384, 136), (333, 72, 1288)]
# each tile size of the product, one and several loads of scales, odd edges on every side
TILES = [(4097, 4104, 264), (4090, 4088, 2312), (4315, 2568, 2568), (4100, 2040, 392), (2001, 2056, 2344), (1499, 1288, 2696),
         (901, 2040, 136), (203, 2056, 2440), (201, 2056, 1096), (34, 5128, 5128)]


@pytest.mark.parametrize("m,n,k", FEW + TILES)
def test_product(m, n, k):
    a, w, g = operands(m + n + k, m, n, k)
    r = whole(g, m, n, 128)
    w8 = rc.quantize_blocks(w.bfloat16(), square=True)
    assert torch.equal(rc.dequantize_blocks(w8).double(), w)
    want = a @ w.t()
    for x in (a.bfloat16(), rc.quantize_blocks(a.bfloat16())):
        assert torch.equal(rc.linear_fp8(x, w8), rounded(want))
        assert torch.equal(rc.linear_fp8(x, w8, residual=r.bfloat16()), rounded(want + r))


@pytest.mark.parametrize("m,n,k", [(3, 4616, 264), (16, 6408, 4104), (70, 264, 1032), (300, 1096, 520), (1400, 2312, 1288), (4100, 520, 2056)])
def test_inputs_gradient(m, n, k):
    dy, w_t, g = operands(m + n + k, m, k, n)
    r = whole(g, m, k, 128)
    w8 = rc.quantize_blocks(w_t.t().contiguous().bfloat16(), square=True, transposed=True)
    want = dy @ w_t.t()
    for res in (None, r):
        dx, dw = rc.linear_fp8_backward(dy.bfloat16(), None, w8, residual=None if res is None else res.bfloat16(), want_dw=False)
        assert dw is None and torch.equal(dx, rounded(want if res is None else want + res))


def test_gradient_against_differences():
    """dx and dw are the derivatives of the product of the values: its change along a direction, which
    is linear in each, so that halves of differences are exact.  dx of up to 128 is exact in bf16."""
    m, n, k = 200, 128, 264
    g = gen(7)
    x, w, dy = whole(g, m, k), whole(g, n, k, 1), whole(g, m, n, 1)
    w8 = rc.quantize_blocks(w.bfloat16(), square=True, transposed=True)
    dx, dw = (t.double() for t in rc.linear_fp8_backward(dy.bfloat16(), rc.quantize_blocks(x.bfloat16()), w8))
    f = lambda a, b: ((a @ b.t()) * dy).sum()  # noqa: E731
    for _ in range(3):
        # near the gradients, so that both changes are far from zero
        u, v = whole(g, m, k) + 2 * (dy @ w).sign(), whole(g, n, k) + 2 * (dy.t() @ x).sign()
        by = float(f(x + u, w) - f(x - u, w)) / 2
        assert by == float((u * dx).sum()) and abs(by) > 100
        by = float(f(x, w + v) - f(x, w - v)) / 2
        assert by == float((v * dw).sum()) and abs(by) > 100


def test_gradient_against_differences_of_ordinary_values():
    """The same along directions near the gradients themselves, of normal values.  dy is what its quantisation
    makes of it, so dx is off by its rounding, 2^-8 relative, by its products' cuts, each below 2^-13 of
    the largest of eight, which is at most the largest |dy| times the largest |w| among them (all
    eights hold normal codes), and by the sums, 2^-23 of the magnitudes a step: one for each 64 of n and the
    8 values in one.  dw is off by its sums alone, a step for each 16 rows and the 16 in one, 64 where shares
    are joined, and its rounding.  All are added as if of one sign."""
    m, n, k = 300, 264, 136
    g = gen(8)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    w8 = rc.quantize_blocks(randn(n, k).bfloat16(), square=True, transposed=True)
    x8, dy8 = rc.quantize_blocks(randn(m, k).bfloat16()), rc.quantize_blocks(randn(m, n).bfloat16())
    xv, wv, dy = (rc.dequantize_blocks(b) for b in (x8, w8, dy8))
    dx, dw = (t.double() for t in rc.linear_fp8_backward(dy, x8, w8))
    xv, wv, dy = xv.double(), wv.double(), dy.double()
    f = lambda a, b: ((a @ b.t()) * dy).sum()  # noqa: E731
    eight = lambda t: torch.nn.functional.pad(t.abs(), (0, -n % 8)).unflatten(1, (-1, 8)).amax(2)  # noqa: E731
    cut = 2.0 ** -13 * 8 * (eight(dy) @ eight(wv.t()).t())   # certain, of each element of dx
    for _ in range(3):
        u, v = dy @ wv + 4 * randn(m, k).double(), dy.t() @ xv + 4 * randn(n, k).double()
        by = float(f(xv + u, wv) - f(xv - u, wv)) / 2
        sums = (n / 64 + 8) * 2.0 ** -23 * (dy.abs() @ wv.abs())
        tol = float((u.abs() * (2.0 ** -8 * (dy @ wv).abs() + (cut + sums) * (1 + 2.0 ** -8))).sum())
        assert tol < 0.1 * abs(by)
        assert abs(by - float((u * dx).sum())) <= tol, (by, tol)
        by = float(f(xv, wv + v) - f(xv, wv - v)) / 2
        tol = (m / 16 + 80) * 2.0 ** -23 * float((v.abs() * (dy.abs().t() @ xv.abs())).sum())
        assert tol < 0.1 * abs(by)
        assert abs(by - float((v * dw).sum())) <= tol, (by, tol)


@pytest.mark.parametrize("plan", WEIGHT_GRADIENTS, ids=str)
def test_weight_gradient(plan):
    """Every kind of plan, over rows none of which is zero; what lies past the rows and columns of
    a strided dy, and what a workspace held, stay out of it."""
    m, n, k = plan[:3]
    need = rc.lib().rc_linear_fp8_backward_workspace_bytes(m, n, k, 0, 1)
    assert need == workspace_bytes(plan)
    g = gen(m + n + k)
    x = whole(g, m, k) * powers(g, m, k, torch.zeros(1, -(-k // 128), dtype=torch.int64, device=DEV), up=2)
    dy = whole(g, m, n)
    want = (dy.t() @ x).float()
    assert float(want.abs().max()) < 2 ** 24
    x8, buf = rc.quantize_blocks(x.bfloat16()), torch.full((m + 64, n + 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    dyb = buf[:m, :n].copy_(dy)
    for ws in (None, torch.full((max(need, 1),), 255, dtype=torch.uint8, device=DEV)):
        dw = torch.full((n, k), float("nan"), device=DEV)
        assert torch.equal(rc.linear_fp8_backward(dyb, x8, None, dw=dw, want_dx=False, workspace=ws)[1], want)
