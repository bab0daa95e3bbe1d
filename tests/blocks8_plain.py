"""Blocks of e4m3 codes by their definition, in 64 bits and on the CPU."""
import torch

BLOCK = 128
E4M3 = torch.float8_e4m3fn


def quantize(x, square=False):
    """(code values [m, k], exponents + 127 [m or its blocks, blocks of k], values [m, k]), fp64."""
    x = x.detach().cpu().double()
    m, k = x.shape
    r = BLOCK if square else 1
    rows, cols = -(-m // r), -(-k // BLOCK)
    full = torch.zeros(rows * r, cols * BLOCK, dtype=torch.float64)
    full[:m, :k] = torch.where(torch.isfinite(x), x.abs(), 0.0)
    top = full.view(rows, r, cols, BLOCK).amax((1, 3))
    frac, e = torch.frexp(top)
    e = torch.where(top > 0, (e - torch.where(frac <= 0.875, 9, 8)).clamp(min=-127), 0)
    at = e.repeat_interleave(r, 0)[:m].repeat_interleave(BLOCK, 1)[:, :k]
    v = torch.where(torch.isfinite(x), x * torch.exp2(-at.double()), torch.nan)
    # float32 holds a bf16 value times a power of two; the conversion rounds to nearest, ties to even
    codes = v.float().to(E4M3).double()
    return codes, (e + 127).to(torch.uint8), codes * torch.exp2(at.double())


def codes_of(b):
    """The code values of Fp8Blocks, fp64 on the CPU."""
    return b.codes[:, :b.shape[1]].contiguous().view(E4M3).cpu().double()


def exps_of(b, square=False):
    e = b.exps[:, :b.shape[0]].t().contiguous().cpu()
    return e[::BLOCK] if square else e


def rows(g, m, k, device="cuda", wide=0):
    """bf16 rows of their own magnitude with a few loud channels; wide: a view of a buffer of that many more columns."""
    x = torch.randn(m, k + wide, generator=g) * torch.exp(0.5 * torch.randn(m, 1, generator=g))
    x = torch.where(torch.rand(1, k + wide, generator=g) < 0.02, 20 * x, x).bfloat16().to(device)
    return x[:, wide:]
