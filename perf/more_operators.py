"""The projections of a layer in 8 bits, as a program calls them.

A layer's projections are most of its arithmetic outside the attention, and
their inputs most of what training keeps for the backward pass.  The operators
measured here hold both as e4m3 codes with one power-of-two scale for each
block of 128 values: the quantisation of activations (blocks of a row) and of
weights (128 x 128 squares, also transposed, for the inputs' gradient), the
product of both, its backward pass, in which the 8-bit activations that the
product has read are the checkpoint for the weights' gradient, and the expansion
of a checkpoint for whoever reads it as bf16.

The scale of a block is 2^e with the smallest e that brings its largest
magnitude to at most 448, the largest e4m3 value (e = 0 for a block of zeros).
Sizes: the layouts' rows, as in operators.py; H heads of D channels.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
BLOCK = 128
MOST = 25152 * 7680 * 2560  # multiplications of the largest listed case


def listed():
    return [
        # a toy model's activations: the launch is all there is
        dict(name="quant_tiny", op="quant", M=80, K=128, wide=False),
        # queries' input of a 1024-pixel step with five references, every row: what a recompute quantises per projection
        dict(name="quant_rows", op="quant", M=25152, K=2560, wide=False),
        # a fused projection's weights, once per load or optimiser step, with the transposed form
        dict(name="quant_weight", op="weight", N=7680, K=2560),
        # a checkpoint back to bf16, odd rows and a last block of 8 channels
        dict(name="expand_ragged", op="expand", M=8771, K=1928),
        # the toy model's fused projection
        dict(name="linear_tiny", op="linear", M=80, N=384, K=128, residual=False, wide=False),
        # two vectors of a guided pair through a projection: reading the weights is all there is
        dict(name="linear_vectors", op="linear", M=2, N=7680, K=2560, residual=False, wide=False),
        # live rows of a 1024-pixel step: output projection and residual, odd prompt length
        dict(name="linear_out", op="linear", M=4315, N=2560, K=2560, residual=True, wide=False),
        # every row of a recompute with five references through the fused projection
        dict(name="linear_full", op="linear", M=25152, N=7680, K=2560, residual=False, wide=False),
        # the toy model's backward pass
        dict(name="bwd_tiny", op="bwd", M=80, N=384, K=128),
        # odd aspect ratios; channels that no block of 128 divides
        dict(name="bwd_ragged", op="bwd", M=4840, N=2568, K=1928),
        # three samples of 512-pixel edits with two references: output projection of a narrow model, few tiles and many rows
        dict(name="bwd_out", op="bwd", M=10944, N=1280, K=1280),
        # two 1024-pixel samples with one reference each, fused projection
        dict(name="bwd_fused", op="bwd", M=17536, N=7680, K=2560),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant", "weight", "expand", "linear", "linear", "linear", "bwd", "bwd", "bwd"])
    n, k = (8 * _log(rng, 1, 960) for _ in range(2))
    if op == "weight":
        return dict(op=op, N=n, K=k)
    if op in ("quant", "expand"):
        c = dict(op=op, M=_log(rng, 1, 30000), K=k)
        return dict(c, wide=rng.random() < 0.4) if op == "quant" else c
    # no more than the largest listed case: its backward pass is two products
    most = MOST // (2 * n * k) if op == "bwd" else MOST // (n * k)
    c = dict(op=op, M=_log(rng, 1, max(1, min(30000, most))), N=n, K=k)
    return dict(c, residual=rng.random() < 0.4, wide=rng.random() < 0.4) if op == "linear" else c


def work(case):
    op, k = case["op"], case["K"]
    if op == "weight":
        return {"bytes": case["N"] * k * 4, "flops": case["N"] * k * 2}
    m = case["M"]
    if op in ("quant", "expand"):
        return {"bytes": m * k * 3 + m * -(-k // BLOCK), "flops": m * k * 2}
    n = case["N"]
    if op == "linear":
        return {"bytes": 2 * m * k + n * k + 2 * m * n * (2 if case["residual"] else 1), "flops": 2 * m * n * k}
    return {"bytes": 2 * m * n + m * k + n * k + 2 * m * k + 4 * n * k, "flops": 4 * m * n * k}


# ---------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _activations(g, m, k, wide=False):
    """Rows of their own magnitude with some channels far above the others;
    wide: a view of a buffer twice as wide."""
    x = torch.randn(m, 2 * k if wide else k, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(m, 1, generator=g, device=DEV))
    loud = torch.rand(1, x.shape[1], generator=g, device=DEV) < 0.01
    x = torch.where(loud, 20 * x, x).to(BF16)
    return x[:, k:] if wide else x


def prepare(case, seed):
    g, op, s = _gen(seed), case["op"], {"case": case}
    if own:
        import paper_2608_21229_amd as rc
    if op != "weight":
        s["x"] = _activations(g, case["M"], case["K"], case.get("wide", False))
    if op in ("weight", "linear", "bwd"):
        s["w"] = (torch.randn(case["N"], case["K"], generator=g, device=DEV) * case["K"] ** -0.5).to(BF16)
    if op == "linear":
        s["residual"] = _activations(g, case["M"], case["N"]) if case["residual"] else None
    if op == "bwd":
        s["dy"] = (_activations(g, case["M"], case["N"]).float() * 1e-3).to(BF16)
    # held in 8 bits by the program: weights since they were loaded, checkpoints since the forward pass
    if op in ("linear", "bwd"):
        s["w_codes"], s["w_exps"] = _quantize(s["w"], True)
        if own:
            s["w8"] = rc.quantize_blocks(s["w"], square=True, transposed=True)
    if op in ("expand", "bwd"):
        s["x_codes"], s["x_exps"] = _quantize(s["x"], False)
        if own:
            s["x8"] = rc.quantize_blocks(s["x"])
        del s["x"]
    return s


# ---------------------------------------------------------------- plain forms
def _spread(e, m, k, square):
    """A block's number at each of its values, [m, k]."""
    e = e.repeat_interleave(BLOCK, 1)[:, :k]
    return e.repeat_interleave(BLOCK, 0)[:m] if square else e


def _pow2(e):
    """2^e in 32 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _quantize(x, square):
    """e4m3 codes [m, k] and the blocks' exponents + 127, [m or its blocks, blocks of k]."""
    m, k = x.shape
    x = x.float()
    a = torch.nn.functional.pad(x.abs(), (0, -k % BLOCK, 0, -m % BLOCK if square else 0))
    a = a.unflatten(1, (-1, BLOCK)).amax(2)
    if square:
        a = a.unflatten(0, (-1, BLOCK)).amax(1)
    frac, e = torch.frexp(a)
    e = torch.where(a > 0, (e - 8 - (frac <= 0.875).int()).clamp(min=-127), 0)
    return (x * _spread(_pow2(-e), m, k, square)).to(F8), (e + 127).to(torch.uint8)


def _values(codes, exps, square=False):
    """What codes stand for, in 32 bits."""
    return codes.float() * _spread(_pow2(exps.int() - 127), *codes.shape, square)


def _run_own(s, case):
    import paper_2608_21229_amd as rc
    op = case["op"]
    if op == "quant":
        x8 = rc.quantize_blocks(s["x"])
        return [x8.codes[:, :case["K"]].view(F8), x8.exps[:, :case["M"]].t()]
    if op == "weight":
        w8 = rc.quantize_blocks(s["w"], square=True, transposed=True)
        return [w8.codes[:, :case["K"]].view(F8), w8.exps[:, :case["N"]:BLOCK].t(), w8.t.codes[:, :case["N"]].view(F8),
                w8.t.exps[:, :case["K"]:BLOCK].t()]
    if op == "expand":
        return [rc.dequantize_blocks(s["x8"])]
    if op == "linear":
        return [rc.linear_fp8(s["x"], s["w8"], residual=s["residual"])]
    return list(rc.linear_fp8_backward(s["dy"], s["x8"], s["w8"]))


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    op = case["op"]
    if op == "quant":
        return list(_quantize(s["x"], False))
    if op == "weight":
        codes, exps = _quantize(s["w"], True)
        return [codes, exps, codes.t().contiguous(), exps.t().contiguous()]
    if op == "expand":
        return [_values(s["x_codes"], s["x_exps"]).to(BF16)]
    w = _values(s["w_codes"], s["w_exps"], True)
    if op == "linear":
        y = torch.matmul(_values(*_quantize(s["x"], False)), w.t())
        return [(y if s["residual"] is None else y + s["residual"].float()).to(BF16)]
    dx = torch.matmul(_values(*_quantize(s["dy"], False)), w).to(BF16)
    return [dx, torch.matmul(s["dy"].float().t(), _values(s["x_codes"], s["x_exps"]))]


# ---------------------------------------------------------------- 64 bits, from the definitions
def _exact_blocks(x, square):
    """The nearest value of the e4m3 grid for each x / 2^e (ties to the even
    one), and e + 127 per block, by search over the 9 powers that can be it."""
    x = x.double()
    m, k = x.shape
    r = BLOCK if square else 1
    rows, cols = -(-m // r), -(-k // BLOCK)
    full = torch.zeros(rows * r, cols * BLOCK, dtype=torch.float64, device=DEV)
    full[:m, :k] = x.abs()
    top = full.view(rows, r, cols, BLOCK).permute(0, 2, 1, 3).reshape(rows, cols, -1).max(2).values
    e = torch.floor(torch.log2(torch.where(top > 0, top, 256.0))) - 12
    for _ in range(9):
        e = torch.where((top > 448 * torch.exp2(e)), e + 1, e)
    e = torch.where(top > 0, e, torch.zeros_like(e)).clamp(min=-127)
    at = e.repeat_interleave(r, 0)[:m].repeat_interleave(BLOCK, 1)[:, :k]
    v = x * torch.exp2(-at)
    step = torch.exp2(torch.frexp(v.abs().clamp(min=2.0 ** -6))[1].double() - 4)
    return torch.round(v / step) * step, (e + 127).to(torch.uint8), at


def _exact_values(x, square):
    v, _, at = _exact_blocks(x, square)
    return v * torch.exp2(at)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "quant":
        return list(_exact_blocks(s["x"], False)[:2])
    if op == "weight":
        v, e, _ = _exact_blocks(s["w"], True)
        return [v, e, v.t().contiguous(), e.t().contiguous()]
    if op in ("expand", "bwd"):  # the codes are the input here
        at = (s["x_exps"].double() - 127).repeat_interleave(BLOCK, 1)[:, :case["K"]]
        x = s["x_codes"].double() * torch.exp2(at)
        if op == "expand":
            return [x]
    w = _exact_values(s["w"], True)
    if op == "linear":
        y = _exact_values(s["x"], False) @ w.t()
        return [y if s["residual"] is None else y + s["residual"].double()]
    return [_exact_values(s["dy"], False) @ w, s["dy"].double().t() @ x]
