"""The layer operators around the reference-cached attention, as a program calls them.

A layer of an in-context diffusion transformer normalises and modulates its
input by the timestep, projects it, normalises and rotates queries and keys by
their (time, height, width) position, attends under the block mask and adds
the gated result to the residual; training it needs each part's gradient.  The
operators measured here are those parts next to the attention and the
projection: the gradient of the masked attention, the rotation of queries and
keys (with their norm) and its gradient, and the gated norm and its gradient.

A layout is named by its segment lengths, as in cases.py: st static text
anchors, lt live text tokens, x target tokens, refs reference lengths.
"""
import math

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16


def listed():
    return [
        # the gradient of a toy model's attention: launches are all there is
        dict(name="attn_bwd_tiny", op="attn_bwd", mask="perref", st=8, lt=16, x=64, refs="64", B=1, H=2, D=64,
             fused=False, dlse=False),
        # training on 512-pixel edits with two references, one sample
        dict(name="attn_bwd_512px", op="attn_bwd", mask="perref", st=64, lt=512, x=1024, refs="1024,1024", B=1, H=24,
             D=128, fused=True, dlse=False),
        # odd aspect ratios and prompt lengths, paper mask, 64-wide heads, a loss that reads the log-sum-exp too
        dict(name="attn_bwd_ragged_d64", op="attn_bwd", mask="paper", st=37, lt=203, x=1577, refs="1600,904,519", B=1,
             H=40, D=64, fused=True, dlse=True),
        # two 1024-pixel samples with one reference each
        dict(name="attn_bwd_1024px", op="attn_bwd", mask="perref", st=64, lt=512, x=4096, refs="4096", B=2, H=24, D=128,
             fused=True, dlse=False),
        # queries and keys of a toy model's live rows
        dict(name="rotary_tiny", op="rotary", B=1, N=80, H=2, axes="16,24,24", D=64, interleaved=True, continuous=False,
             norm=False, floats=False, span=64, theta=10000.0),
        # the live rows of a 1024-pixel step, with the per-head norm, from the fused projection
        dict(name="rotary_step", op="rotary", B=1, N=4608, H=24, axes="16,56,56", D=128, interleaved=True,
             continuous=False, norm=True, floats=False, span=64, theta=10000.0),
        # gradient for a short 480-pixel video: halves paired, one frequency ladder over the axes, fractional times, two samples
        dict(name="rotary_bwd_video", op="rotary_bwd", B=2, N=7801, H=12, axes="32,48,48", D=128, interleaved=False,
             continuous=True, norm=True, floats=True, span=4000, theta=1000000.0),
        # gradient without a norm, 64-wide heads of which the last 8 channels do not rotate
        dict(name="rotary_bwd_d64", op="rotary_bwd", B=1, N=1029, H=16, axes="8,24,24", D=64, interleaved=True,
             continuous=False, norm=False, floats=False, span=64, theta=10000.0),
        # the toy model's first norm of live rows
        dict(name="norm_tiny", op="norm", st=0, lt=16, x=64, refs="", B=1, C=128, kind="layer", weight=False, branch=False,
             gate=False, post=False, rscale=1.0),
        # between attention and the next block of a 1024-pixel step
        dict(name="norm_step", op="norm", st=0, lt=512, x=4096, refs="", B=1, C=2560, kind="layer", weight=False,
             branch=True, gate=True, post=False, rscale=1.0),
        # training on 1024-pixel edits: live rows modulated by the timestep, static ones by timestep 0
        dict(name="norm_bwd_1024px", op="norm_bwd", st=64, lt=512, x=4096, refs="4096", B=1, C=2560, kind="layer",
             weight=False, branch=True, gate=True, post=False, rscale=1.0),
        # norms before and after the block, with weights, odd lengths, two samples
        dict(name="norm_bwd_sandwich", op="norm_bwd", st=37, lt=203, x=1577, refs="1600,519", B=2, C=1928, kind="rms",
             weight=True, branch=True, gate=True, post=True, rscale=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn_bwd", "attn_bwd", "rotary", "rotary_bwd", "norm", "norm_bwd"])
    if op == "attn_bwd":
        refs = [_log(rng, 1, 3000) for _ in range(rng.randint(1, 3))]
        c = dict(op=op, mask=rng.choice(["perref", "paper", "isolated", "dense"]), st=_log(rng, 1, 128),
                 lt=_log(rng, 1, 800), x=_log(rng, 1, 4096), refs=",".join(map(str, refs)), B=rng.randint(1, 2),
                 H=_log(rng, 1, 24), D=rng.choice([64, 128]), fused=rng.random() < 0.7, dlse=rng.random() < 0.3)
        # no more than the largest listed case, whose plain form holds a few [B, H, N, N] tensors
        c["H"] = max(1, min(c["H"], int(2 * 24 * 8768 ** 2 / (c["B"] * _rows(c) ** 2))))
        return c
    if op in ("rotary", "rotary_bwd"):
        D = rng.choice([64, 128])
        pairs = rng.choice([D // 2, D // 2, 3 * D // 8])
        h = rng.randint(4, pairs // 2 - 2)
        axes = [2 * (pairs - 2 * h), 2 * h, 2 * h]
        return dict(op=op, B=rng.randint(1, 2), N=_log(rng, 1, 8192), H=_log(rng, 1, 16), axes=",".join(map(str, axes)),
                    D=D, interleaved=rng.random() < 0.6, continuous=rng.random() < 0.4, norm=rng.random() < 0.7,
                    floats=rng.random() < 0.3, span=_log(rng, 64, 100000), theta=rng.choice([10000.0, 1000000.0]))
    branch = rng.random() < 0.8
    return dict(op=op, st=rng.choice([0, _log(rng, 1, 128)]), lt=_log(rng, 1, 800), x=_log(rng, 1, 4096),
                refs=",".join(str(_log(rng, 1, 2000)) for _ in range(rng.randint(0, 2))), B=rng.randint(1, 2),
                C=8 * _log(rng, 8, 480), kind=rng.choice(["layer", "rms"]), weight=rng.random() < 0.4, branch=branch,
                gate=branch and rng.random() < 0.8, post=branch and rng.random() < 0.4, rscale=rng.choice([1.0, 0.5]))


# ---------------------------------------------------------------- layouts
def _refs(case):
    return [int(r) for r in case["refs"].split(",") if r]


def _segments(case):
    """(kind, length) of each segment; kinds 0 anchors, 1 text, 2 target, 3 reference."""
    segs = [(0, case["st"]), (1, case["lt"]), (2, case["x"])] + [(3, r) for r in _refs(case)]
    return [(k, n) for k, n in segs if n > 0]


def _reads(mask, i, a, j, b):
    """Whether segment i of kind a reads segment j of kind b."""
    if mask == "dense":
        return True
    live = a in (1, 2)
    if mask == "paper":
        return b != 0 if live else b in (0, 3)
    if mask == "isolated":
        return a != 0 and (b != 0 if live else b == 3)
    return live or b == 0 or (a == 3 and i == j)


def _visible(case):
    segs = _segments(case)
    return [[_reads(case["mask"], i, a, j, b) for j, (b, _) in enumerate(segs)] for i, (a, _) in enumerate(segs)]


def _pairs(case):
    lens = [n for _, n in _segments(case)]
    return sum(n * m for n, row in zip(lens, _visible(case)) for m, see in zip(lens, row) if see)


def _rows(case):
    return sum(n for _, n in _segments(case))


def _spans(case):
    """(rows, modulation group): live rows take group 0, static ones group 1."""
    return [(n, 0 if k in (1, 2) else 1) for k, n in _segments(case)]


def _groups(case):
    return 1 + max(g for _, g in _spans(case))


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def _turns(case, device=None):
    """Per rotated pair: its axis and its angle per unit of position (radians)."""
    axes, theta = _axes(case), case["theta"]
    width = sum(axes)
    axis, freq = [], []
    for a, d in enumerate(axes):
        for i in range(d // 2):
            axis.append(a)
            e = 2.0 * (len(axis) - 1) / width if case["continuous"] else 2.0 * i / d
            freq.append(theta ** -e)
    return torch.tensor(axis, device=device), torch.tensor(freq, dtype=torch.float64, device=device)


def work(case):
    op = case["op"]
    if op == "attn_bwd":
        rows = case["B"] * _rows(case) * case["H"]
        return {"bytes": rows * (8 * case["D"] * 2 + (8 if case["dlse"] else 4)),
                "flops": 10 * case["D"] * _pairs(case) * case["B"] * case["H"]}
    if op in ("rotary", "rotary_bwd"):
        values = 2 * case["B"] * case["N"] * case["H"] * case["D"]
        passes = 3 if op == "rotary_bwd" and case["norm"] else 2
        return {"bytes": values * 2 * passes + case["N"] * 4 * len(_axes(case)), "flops": values * 8}
    values = case["B"] * _rows(case) * case["C"]
    if op == "norm":
        return {"bytes": values * 2 * (4 if case["branch"] else 2), "flops": values * 10}
    return {"bytes": values * 2 * (6 if case["branch"] else 4), "flops": values * 20}


# ---------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(BF16)


def _seen(case, n):
    """[N, N] truth values: row reads column."""
    segs = _segments(case)
    ids = torch.repeat_interleave(torch.arange(len(segs), device=DEV), torch.tensor([m for _, m in segs], device=DEV),
                                  output_size=n)
    return torch.tensor(_visible(case), device=DEV)[ids][:, ids]


def prepare(case, seed):
    g, op, s = _gen(seed), case["op"], {"case": case}
    if op == "attn_bwd":
        B, H, D, N = case["B"], case["H"], case["D"], _rows(case)
        if case["fused"]:  # views of one fused projection
            qkv = _randn(g, B, N, 3, H, D)
            s["q"], s["k"], s["v"] = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        else:
            s["q"], s["k"], s["v"] = (_randn(g, B, N, H, D) for _ in range(3))
        s["seen"] = _seen(case, N)
        # the forward pass, whose output and log-sum-exp training keeps
        q, k, v = (t.float().transpose(1, 2).contiguous() for t in (s["q"], s["k"], s["v"]))
        sc = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).masked_fill_(~s["seen"], -math.inf)
        s["lse"] = torch.logsumexp(sc, 3)
        p = sc.sub_(s["lse"].clamp(min=-1e30).unsqueeze(3)).exp_()
        s["o"] = torch.matmul(p, v).transpose(1, 2).to(BF16).contiguous()
        del sc, p
        s["do"] = _randn(g, B, N, H, D)
        s["dlse"] = torch.randn(B, H, N, generator=g, device=DEV) if case["dlse"] else None
        if own:
            import paper_2608_21229_amd as rc
            s["layout"] = rc.Layout(_segments(case), case["mask"])
    elif op in ("rotary", "rotary_bwd"):
        B, N, H, D = case["B"], case["N"], case["H"], case["D"]
        qkv = _randn(g, B, N, 3, H, D, std=1.5)
        s["q"], s["k"] = qkv[:, :, 0], qkv[:, :, 1]
        half = case["span"] // 2
        s["pos"] = torch.randint(-half, half, (N, len(_axes(case))), generator=g, device=DEV, dtype=torch.int32)
        if case["floats"]:
            s["pos"] = s["pos"].float() * 0.25
        s["wq"] = (1 + _randn(g, D, std=0.2)) if case["norm"] else None
        s["wk"] = (1 + _randn(g, D, std=0.2)) if case["norm"] else None
        if op == "rotary_bwd":
            s["dq"], s["dk"] = _randn(g, B, N, H, D), _randn(g, B, N, H, D)
        s["axis"], s["freq"] = _turns(case, DEV)
        if own:
            import paper_2608_21229_amd as rc
            s["rotary"] = rc.Rotary(D, _axes(case), theta=case["theta"], interleaved=case["interleaved"],
                                    continuous=case["continuous"])
    else:
        B, N, C, G = case["B"], _rows(case), case["C"], _groups(case)
        s["spans"] = _spans(case)
        s["group"] = torch.repeat_interleave(torch.tensor([k for _, k in s["spans"]], device=DEV),
                                             torch.tensor([n for n, _ in s["spans"]], device=DEV), output_size=N)
        s["h"] = _randn(g, B, N, C, std=2.0)
        s["x"] = _randn(g, B, N, C) if case["branch"] else None
        mod = _randn(g, B, G, 3 * C, std=0.5)  # one projection of the timestep's embedding
        s["shift"], s["scale"], s["gate"] = mod[..., :C], mod[..., C:2 * C], mod[..., 2 * C:] if case["gate"] else None
        s["w"] = (1 + _randn(g, C, std=0.2)) if case["weight"] else None
        s["wp"] = (1 + _randn(g, C, std=0.2)) if case["post"] else None
        if op == "norm_bwd":
            s["dy"], s["dh"] = _randn(g, B, N, C), _randn(g, B, N, C)
    return s


# ---------------------------------------------------------------- plain forms
def _attn_bwd(s, case, t):
    """t: the working precision."""
    scale = 1.0 / math.sqrt(case["D"])
    q, k, v, o, do = (s[n].to(t).transpose(1, 2).contiguous() for n in ("q", "k", "v", "o", "do"))
    p = torch.matmul(q, k.transpose(2, 3)).mul_(scale).sub_(s["lse"].to(t).unsqueeze(3)).exp_()
    p.masked_fill_(~s["seen"], 0.0)
    delta = (do * o).sum(3, keepdim=True)
    if s["dlse"] is not None:
        delta = delta - s["dlse"].to(t).unsqueeze(3)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_(delta).mul_(p)
    dq, dk = torch.matmul(ds, k) * scale, torch.matmul(ds.transpose(2, 3), q) * scale
    return [x.transpose(1, 2).contiguous() for x in (dq, dk, dv)]


def _cos_sin(s, case, t):
    """[N, 1, pairs] each; the angles in 64 bits, since far positions lose them in 32."""
    angle = s["pos"].double()[:, s["axis"]] * s["freq"]
    return angle.cos().to(t).unsqueeze(1), angle.sin().to(t).unsqueeze(1)


def _turn(x, cos, sin, interleaved):
    """x [B, N, H, D] with its pairs turned; channels past the rotated width stay."""
    half = cos.shape[-1]
    w, rest = x[..., : 2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = w[..., 0::2], w[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)
    a, b = w[..., :half], w[..., half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


def _rotary(s, case, t):
    cos, sin = _cos_sin(s, case, t)
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        x = x.to(t)
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.to(t)
        out.append(_turn(x, cos, sin, case["interleaved"]))
    return out


def _rotary_bwd(s, case, t):
    cos, sin = _cos_sin(s, case, t)
    out, dw = [], []
    for g, x, w in ((s["dq"], s["q"], s["wq"]), (s["dk"], s["k"], s["wk"])):
        u = _turn(g.to(t), cos, -sin, case["interleaved"])
        if w is not None:
            x = x.to(t)
            r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
            xh = x * r
            dw.append((u * xh).sum((0, 1, 2)))
            u = u * w.to(t)
            u = r * (u - xh * (u * xh).mean(-1, keepdim=True))
        out.append(u)
    return out, dw


def _normed(h, kind):
    """The normalised rows and their reciprocal deviation."""
    if kind == "layer":
        h = h - h.mean(-1, keepdim=True)
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)
    return h * r, r


def _back(dn, n, r, kind):
    """Gradient through the norm."""
    out = dn - n * (dn * n).mean(-1, keepdim=True)
    return r * (out - dn.mean(-1, keepdim=True) if kind == "layer" else out)


def _of_rows(s, name, t):
    return s[name].to(t)[:, s["group"]]


def _norm(s, case, t):
    h = s["h"].to(t)
    out = []
    if case["branch"]:
        u = s["x"].to(t)
        if case["post"]:
            u = _normed(u, "rms")[0] * s["wp"].to(t)
        if case["gate"]:
            u = u * _of_rows(s, "gate", t)
        h = h + case["rscale"] * u
        out.append(h)
    n, _ = _normed(h, case["kind"])
    if case["weight"]:
        n = n * s["w"].to(t)
    out.append(n * (1 + _of_rows(s, "scale", t)) + _of_rows(s, "shift", t))
    return out


def _norm_bwd(s, case, t):
    """Gradients of the rows, and of what is shared between rows."""
    dy, scale = s["dy"].to(t), 1 + _of_rows(s, "scale", t)
    n, r = _normed(s["h"].to(t), case["kind"])
    pick = torch.nn.functional.one_hot(s["group"], _groups(case)).to(t).t().contiguous()  # [G, N]
    rows, shared = [], []
    w = s["w"].to(t) if case["weight"] else 1.0
    shared += [torch.matmul(pick, dy), torch.matmul(pick, dy * n * w)]
    if case["weight"]:
        shared.append((dy * scale * n).sum((0, 1)))
    dh = s["dh"].to(t) + _back(dy * scale * w, n, r, case["kind"])
    rows.append(dh)
    if case["branch"]:
        gate = _of_rows(s, "gate", t) if case["gate"] else 1.0
        du, x = case["rscale"] * dh * gate, s["x"].to(t)
        u = x
        if case["post"]:
            xn, xr = _normed(x, "rms")
            u = xn * s["wp"].to(t)
            shared.append((du * xn).sum((0, 1)))
            du = _back(du * s["wp"].to(t), xn, xr, "rms")
        if case["gate"]:
            shared.append(torch.matmul(pick, case["rscale"] * dh * u))
        rows.append(du)
    return rows, shared


def _run_own(s, case):
    import paper_2608_21229_amd as rc
    op = case["op"]
    if op == "attn_bwd":
        return list(rc.full_attention_backward(s["layout"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"],
                                               dlse=s["dlse"]))
    if op == "rotary":
        return list(rc.qk_rotary(s["rotary"], s["q"], s["k"], s["pos"], q_norm=s["wq"], k_norm=s["wk"]))
    if op == "rotary_bwd":
        a, b, da, db = rc.qk_rotary_backward(s["rotary"], s["dq"], s["dk"], s["pos"], q=s["q"], k=s["k"],
                                             q_norm=s["wq"], k_norm=s["wk"])
        return [a, b] + ([da, db] if case["norm"] else [])
    if op == "norm":
        h, y = rc.gated_norm(s["h"], s["x"], gate=s["gate"], scale=s["scale"], shift=s["shift"], weight=s["w"],
                             post_weight=s["wp"], norm=case["kind"], spans=s["spans"], residual_scale=case["rscale"])
        return [h, y] if case["branch"] else [y]
    d = rc.gated_norm_backward(s["dy"], s["h"], s["x"], dh=s["dh"], gate=s["gate"], scale=s["scale"], shift=s["shift"],
                               weight=s["w"], post_weight=s["wp"], norm=case["kind"], spans=s["spans"],
                               residual_scale=case["rscale"])
    return ([d.h] + ([d.x] if case["branch"] else []) + [d.shift, d.scale] + ([d.weight] if case["weight"] else [])
            + ([d.post_weight] if case["post"] else []) + ([d.gate] if case["gate"] else []))


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    t, op = torch.float32, case["op"]
    if op == "attn_bwd":
        return [x.to(BF16) for x in _attn_bwd(s, case, t)]
    if op == "rotary":
        return [x.to(BF16) for x in _rotary(s, case, t)]
    if op == "norm":
        return [x.to(BF16) for x in _norm(s, case, t)]
    rows, shared = (_rotary_bwd if op == "rotary_bwd" else _norm_bwd)(s, case, t)
    return [x.to(BF16) for x in rows] + shared


# ---------------------------------------------------------------- 64 bits, from the definitions
def _exact_attn(s, case):
    """Per batch entry and head, with the softmax's Jacobian written out row by row of blocks."""
    B, H, D, N = case["B"], case["H"], case["D"], _rows(case)
    scale = 1.0 / math.sqrt(D)
    grads = [torch.zeros(B, N, H, D, dtype=torch.float64, device=DEV) for _ in range(3)]
    for b in range(B):
        for h in range(H):
            q, k, v, o, do = (s[n][b, :, h].double() for n in ("q", "k", "v", "o", "do"))
            for i in range(0, N, 4096):
                at = slice(i, min(N, i + 4096))
                p = torch.where(s["seen"][at], torch.exp(scale * (q[at] @ k.t()) - s["lse"][b, h, at, None].double()), 0.0)
                mean = (do[at] * o[at]).sum(1)
                if s["dlse"] is not None:
                    mean = mean - s["dlse"][b, h, at].double()
                ds = scale * p * (do[at] @ v.t() - mean[:, None])
                grads[0][b, at, h] = ds @ k
                grads[1][b, :, h] += ds.t() @ q[at]
                grads[2][b, :, h] += p.t() @ do[at]
    return grads


def _unit(s, case):
    """The turns as complex numbers of length one, [N, 1, pairs]."""
    angle = torch.stack([s["pos"][:, a].double() * f for a, f in zip(s["axis"].tolist(), s["freq"].tolist())], 1)
    return torch.polar(torch.ones_like(angle), angle).unsqueeze(1)


def _complex_turn(x, unit, interleaved):
    half = unit.shape[-1]
    first = x[..., : 2 * half]
    pairs = first.unflatten(-1, (half, 2)) if interleaved else first.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * half:]], -1)


def _exact_rotary(s, case, back):
    unit, out, dw = _unit(s, case), [], []
    for x, w, g in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x = x.double().requires_grad_(back)
        weight = w.double().requires_grad_(back) if w is not None else None
        z = x if w is None else weight * x / (x.pow(2).sum(-1, keepdim=True) / case["D"] + 1e-6).sqrt()
        y = _complex_turn(z, unit, case["interleaved"])
        if not back:
            out.append(y)
            continue
        got = torch.autograd.grad(y, [x] + ([weight] if w is not None else []), g.double())
        out.append(got[0])
        dw += got[1:]
    return out + dw


def _exact_norm(s, case, back):
    """The forward pass by the definition; its gradient by differentiation."""
    rows = {n: s[n].double().requires_grad_(back) for n in ("h", "x", "shift", "scale", "gate", "w", "wp")
            if s[n] is not None}
    of = lambda n: rows[n].index_select(1, s["group"])  # noqa: E731
    h, out = rows["h"], []
    if case["branch"]:
        u = rows["x"]
        if case["post"]:
            u = rows["wp"] * u / (u.pow(2).sum(-1, keepdim=True) / case["C"] + 1e-6).sqrt()
        if case["gate"]:
            u = of("gate") * u
        u = case["rscale"] * u
        h = h + u
        out.append(h)
    # the gradient is taken where the rows after the residual are the given ones
    at = rows["h"] if back else h
    c = at - (at.sum(-1, keepdim=True) / case["C"] if case["kind"] == "layer" else 0.0)
    n = c / (c.pow(2).sum(-1, keepdim=True) / case["C"] + 1e-6).sqrt()
    if case["weight"]:
        n = n * rows["w"]
    y = n * (1 + of("scale")) + of("shift")
    if not back:
        return out + [y]
    want = ["shift", "scale"] + (["w"] if case["weight"] else [])
    got = torch.autograd.grad(y, [rows["h"]] + [rows[n] for n in want], s["dy"].double())
    dh, shared = got[0] + s["dh"].double(), list(got[1:])
    if not case["branch"]:
        return [dh] + shared
    want = (["wp"] if case["post"] else []) + (["gate"] if case["gate"] else [])
    got = torch.autograd.grad(u, [rows["x"]] + [rows[n] for n in want], dh)
    return [dh, got[0]] + shared + list(got[1:])


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "attn_bwd":
        return _exact_attn(s, case)
    if op in ("rotary", "rotary_bwd"):
        return _exact_rotary(s, case, op == "rotary_bwd")
    return _exact_norm(s, case, op == "norm_bwd")
