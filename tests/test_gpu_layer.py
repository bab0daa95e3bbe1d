"""Rotation of queries and keys and the gated norm, with their gradients,
against their formulas in 64 bits.

Bounds.  An output is rounded once to bf16: half a step, 2^-8 of its value.
The arithmetic before it is fp32: a few 2^-24 of the terms that are summed,
sums over a row of up to 2^12 channels included (pairwise over lanes), the
hardware's sine and cosine of a reduced angle (2^-18 absolute allowed here),
reciprocal square roots (2^-22): 2^-16 of the absolute terms covers them.
Shared gradients are fp32 sums over R rows: 2^-16 of the sum of the absolute
terms covers both the terms and the sum's order (R 2^-24 at most 2^-11 in the
worst case, but the partial sums here are of at most 64 rows at a time)."""
import pytest
import torch

import paper_2608_21229_amd as rc
from synthgen import bf16_normal, derive_seed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, F = 2.0 ** -8, 2.0 ** -16
BF16 = torch.bfloat16


def draw(shape, seed, i, std=1.0):
    return bf16_normal(tuple(shape), derive_seed(seed, 0, 0, i), std).to(DEV)


def inside(name, got, ref, tol):
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.isfinite(got).all(), name
    over = ((got.double() - ref).abs() / (tol + 1e-30)).max().item() if ref.numel() else 0.0
    print(f"[layer] {name} err/bound={over:.3f}", flush=True)
    assert over <= 1.0, (name, over)


# ---------------------------------------------------------------- rotation
def _angles(axes, theta, continuous, pos):
    width, p, cols = sum(axes), 0, []
    for a, d in enumerate(axes):
        for i in range(d // 2):
            e = 2.0 * p / width if continuous else 2.0 * i / d
            cols.append(pos[..., a].double() * theta ** -e)
            p += 1
    t = torch.stack(cols, -1) if cols else torch.zeros(*pos.shape[:-1], 0, dtype=torch.float64, device=pos.device)
    t = t.unsqueeze(-2)
    return t if pos.dim() == 3 else t.unsqueeze(0)


def _turned(x, t, interleaved):
    """The rotation and, per channel, the sum of its terms' magnitudes."""
    half = t.shape[-1]
    w, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (w[..., 0::2], w[..., 1::2]) if interleaved else (w[..., :half], w[..., half:])
    c, s = t.cos(), t.sin()
    both = [(a * c - b * s, a * s + b * c), (a.abs() + b.abs(),) * 2]
    out = []
    for u, v in both:
        out.append(torch.cat([torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1), rest], -1))
    return out[0], out[1].abs()


def _rotary_case(D, axes, interleaved, continuous, B, N, H, seed, norm=True, floats=False, batch_pos=False, span=64,
                 theta=10000.0, fused=True):
    R = rc.Rotary(D, axes, theta=theta, interleaved=interleaved, continuous=continuous)
    if fused:
        qkv = draw((B, N, 3, H, D), seed, 0, 1.5)
        q, k = qkv[:, :, 0], qkv[:, :, 1]
    else:
        q, k = draw((B, N, H, D), seed, 0, 1.5), draw((B, N, H, D), seed, 1, 1.5)
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(-span, span, ((B, N) if batch_pos else (N,)) + (len(axes),), generator=g, dtype=torch.int32)
    pos = (pos.float() * 0.37 if floats else pos).to(DEV)
    wq, wk = (1 + draw((D,), seed, 2, 0.3), 1 + draw((D,), seed, 3, 0.3)) if norm else (None, None)
    return R, q, k, pos, wq, wk, _angles(axes, theta, continuous, pos)


def _check_rotary(*args, **kw):
    R, q, k, pos, wq, wk, t = _rotary_case(*args, **kw)
    got = rc.qk_rotary(R, q, k, pos, q_norm=wq, k_norm=wk)
    inter = args[2]
    for name, x, w, y in (("q", q, wq, got[0]), ("k", k, wk, got[1])):
        z = x.double()
        if w is not None:
            z = z * torch.rsqrt(z.square().mean(-1, keepdim=True) + 1e-6) * w.double()
        ref, size = _turned(z, t, inter)
        inside(name, y, ref, U * ref.abs() + F * size)
    return R, q, k, pos, wq, wk, t, got


@pytest.mark.parametrize("D,axes", [(64, (16, 24, 24)), (128, (16, 56, 56)), (128, (32, 48)), (64, (8, 20, 20)),
                                    (128, (0, 64, 32)), (64, (64,))])
@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
@pytest.mark.parametrize("interleaved", [True, False], ids=["pairs", "halves"])
def test_rotation(D, axes, interleaved, norm):
    _check_rotary(D, axes, interleaved, False, 2, 37, 5, seed=3, norm=norm)
    _check_rotary(D, axes, interleaved, True, 1, 70, 3, seed=4, norm=norm, floats=True, batch_pos=True, fused=False)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 63, 257])
@pytest.mark.parametrize("H", [1, 2, 7, 24])
def test_rotation_of_token_and_head_counts(N, H):
    _check_rotary(128, (16, 56, 56), True, False, 1, N, H, seed=N + H)
    _check_rotary(64, (16, 16, 16), False, False, 2, N, H, seed=N + H, norm=False)


@pytest.mark.parametrize("span", [1000, 100_000, 2_000_000_000])
def test_rotation_at_far_positions(span):
    _check_rotary(128, (16, 56, 56), True, False, 1, 50, 2, seed=5, span=span)
    _check_rotary(64, (32, 32), False, True, 1, 50, 2, seed=6, span=span, theta=1e6, norm=False)


def test_rotation_in_place_and_alone():
    R, q, k, pos, wq, wk, _, got = _check_rotary(128, (16, 56, 56), False, False, 2, 33, 6, seed=7)
    a, none = rc.qk_rotary(R, q, None, pos, q_norm=wq)
    none2, b = rc.qk_rotary(R, None, k, pos, k_norm=wk)
    assert none is None and none2 is None and torch.equal(a, got[0]) and torch.equal(b, got[1])
    one, other = rc.qk_rotary(R, q, k, pos, q_norm=wq)  # only queries have a norm
    plain = rc.qk_rotary(R, q, k, pos)
    assert torch.equal(one, got[0]) and torch.equal(other, plain[1])
    c, d = rc.qk_rotary(R, q, k, pos, q_norm=wq, k_norm=wk, q_out=q, k_out=k)
    assert c is q and d is k and torch.equal(q, got[0]) and torch.equal(k, got[1])


def test_rotation_of_no_tokens():
    R = rc.Rotary(64, (16, 24, 24))
    q = torch.empty(1, 0, 2, 64, dtype=BF16, device=DEV)
    a, b = rc.qk_rotary(R, q, q, torch.empty(0, 3, dtype=torch.int32, device=DEV))
    assert a.shape == q.shape and b.shape == q.shape
    w = torch.ones(64, dtype=BF16, device=DEV)
    *_, dw, none = rc.qk_rotary_backward(R, q, q, torch.empty(0, 3, dtype=torch.int32, device=DEV), q=q, q_norm=w)
    assert (dw == 0).all() and none is None


def _check_rotary_backward(*args, **kw):
    R, q, k, pos, wq, wk, t = _rotary_case(*args, **kw)
    seed = kw["seed"]
    dq, dk = draw(q.shape, seed, 8), draw(k.shape, seed, 9)
    got = rc.qk_rotary_backward(R, dq, dk, pos, q=q, k=k, q_norm=wq, k_norm=wk)
    for name, x, w, g, y, dw in (("dq", q, wq, dq, got[0], got[2]), ("dk", k, wk, dk, got[1], got[3])):
        u, size = _turned(g.double(), -t, args[2])
        if w is None:
            inside(name, y, u, U * u.abs() + F * size)
            assert dw is None
            continue
        z = x.double()
        r = torch.rsqrt(z.square().mean(-1, keepdim=True) + 1e-6)
        xh = z * r
        uw = u * w.double()
        ref = r * (uw - xh * (uw * xh).mean(-1, keepdim=True))
        big = r * (size * w.double().abs() + xh.abs() * (size * w.double().abs() * xh.abs()).mean(-1, keepdim=True))
        inside(name, y, ref, U * ref.abs() + F * big)
        inside(name + "_norm", dw, (u * xh).sum((0, 1, 2)), F * (size * xh.abs()).sum((0, 1, 2)))
    return R, q, k, pos, wq, wk, dq, dk, got


@pytest.mark.parametrize("D,axes", [(64, (16, 24, 24)), (128, (16, 56, 56)), (64, (8, 20, 20))])
@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
@pytest.mark.parametrize("interleaved", [True, False], ids=["pairs", "halves"])
def test_rotation_gradient(D, axes, interleaved, norm):
    for N, H in ((1, 1), (37, 5), (300, 24)):
        _check_rotary_backward(D, axes, interleaved, False, 2, N, H, seed=11, norm=norm, fused=N != 37)


def test_rotation_gradient_in_place_and_repeated():
    R, q, k, pos, wq, wk, dq, dk, got = _check_rotary_backward(128, (16, 56, 56), True, False, 1, 1500, 8, seed=12)
    again = rc.qk_rotary_backward(R, dq, dk, pos, q=q, k=k, q_norm=wq, k_norm=wk)
    for a, b in zip(got, again):
        assert torch.equal(a, b)
    only = rc.qk_rotary_backward(R, dq, dk, pos, k=k, k_norm=wk)
    assert torch.equal(only[1], got[1]) and torch.equal(only[3], got[3]) and only[2] is None
    out = rc.qk_rotary_backward(R, dq, dk, pos, q=q, k=k, q_norm=wq, k_norm=wk, dq_out=dq, dk_out=dk)
    assert out[0] is dq
    for a, b in zip(got, out):
        assert torch.equal(a, b)


def test_rotation_gradient_against_differences():
    R, q, k, pos, wq, wk, t = _rotary_case(64, (16, 24, 24), False, False, 1, 9, 2, seed=13)
    dq = draw(q.shape, 13, 8)
    got, _, dw, _ = rc.qk_rotary_backward(R, dq, None, pos, q=q, q_norm=wq)

    def value(x, w):
        z = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        return (_turned(z, t, False)[0] * dq.double()).sum()

    g = torch.Generator().manual_seed(2)
    x, w = q.double(), wq.double()
    for i in range(3):
        sx = torch.randn(x.shape, generator=g, dtype=torch.float64).to(DEV)
        sw = torch.randn(w.shape, generator=g, dtype=torch.float64).to(DEV)
        e = 1e-5
        diff = (value(x + e * sx, w + e * sw) - value(x - e * sx, w - e * sw)) / (2 * e)
        along = (got.double() * sx).sum() + (dw.double() * sw).sum()
        scale = (got.double() * sx).norm() + (dw.double() * sw).norm()  # rounding: U per term, random in sign
        assert abs((along - diff).item()) <= 4 * U * scale.item()


# ---------------------------------------------------------------- gated norm
def _norm_case(B, spans, C, seed, branch=True, gate=True, mod=True, weight=False, post=False, ld=0):
    N, G = sum(n for n, _ in spans), 1 + max(g for _, g in spans)
    rows = lambda i, s=1.0: draw((B, N, C + ld), seed, i, s)[..., :C]  # noqa: E731
    m = draw((B, G, 3 * C), seed, 5, 0.5)
    return dict(h=rows(0, 2.0) + 0.5, x=rows(1) if branch else None,
                gate=m[..., :C] if branch and gate else None, scale=m[..., C:2 * C] if mod else None,
                shift=m[..., 2 * C:] if mod else None, weight=1 + draw((C,), seed, 6, 0.3) if weight else None,
                post_weight=1 + draw((C,), seed, 7, 0.3) if branch and post else None, spans=spans)


def _d(t):
    return None if t is None else t.double()


def _of(t, spans):
    if t is None:
        return None
    return t.double()[:, torch.repeat_interleave(torch.tensor([g for _, g in spans]),
                                                 torch.tensor([n for n, _ in spans])).to(DEV)]


def _residual(c, rs, post_norm, eps):
    """h' and the magnitude of its terms."""
    h = c["h"].double()
    if c["x"] is None:
        return h, h.abs()
    u = c["x"].double()
    if post_norm or c["post_weight"] is not None:
        u = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + eps)
    if c["post_weight"] is not None:
        u = u * c["post_weight"].double()
    g = _of(c["gate"], c["spans"])
    u = rs * (u if g is None else u * g)
    return h + u, h.abs() + u.abs()


def _n(h, kind, eps):
    c = h - h.mean(-1, keepdim=True) if kind == "layer" else h
    r = torch.rsqrt(c.square().mean(-1, keepdim=True) + eps)
    return c * r, r


def _check_norm(c, kind, rs=1.0, post_norm=False, eps=1e-6):
    gh, gy = rc.gated_norm(**c, norm=kind, residual_scale=rs, post_norm=post_norm, eps=eps)
    h, size = _residual(c, rs, post_norm, eps)
    if c["x"] is None:
        assert gh is c["h"]
    else:
        inside("h", gh, h, U * h.abs() + F * size)
    n, r = _n(h, kind, eps)
    w = 1.0 if c["weight"] is None else c["weight"].double()
    s = 1.0 if c["scale"] is None else 1 + _of(c["scale"], c["spans"])
    b = 0.0 if c["shift"] is None else _of(c["shift"], c["spans"])
    ref = n * w * s + b
    # an error of 2^-16 of the row's terms in h', through the norm
    row = (r * (size + size.mean(-1, keepdim=True)) + n.abs() * (n.abs() * r * size).mean(-1, keepdim=True))
    one = torch.ones_like(n)
    inside("y", gy, ref, U * ref.abs() + F * ((row + n.abs()) * (w * one).abs() * ((s - 1) * one).abs().add(1) + (b * one).abs()))
    return gh, gy


SPANS = [(16, 0), (1, 1), (40, 0), (7, 2)]


@pytest.mark.parametrize("C", [8, 64, 128, 504, 512, 520, 1024, 1152, 1928, 2048, 2560, 3080, 4096, 4104, 8192, 16384])
def test_norm_of_widths(C):
    _check_norm(_norm_case(2, SPANS, C, seed=C), "layer")
    _check_norm(_norm_case(1, [(5, 0)], C, seed=C + 1, weight=True, post=True), "rms", rs=0.5)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("parts", [dict(branch=False), dict(gate=False), dict(mod=False), dict(post=True),
                                   dict(weight=True, post=True), dict(weight=True, mod=False, gate=False)],
                         ids=lambda p: "-".join(p))
def test_norm_parts(parts, kind):
    c = _norm_case(2, SPANS, 640, seed=21, ld=24, **parts)
    _check_norm(c, kind, rs=0.7, eps=1e-5)
    if c["x"] is not None:
        _check_norm(c, kind, post_norm=True)
        gh, none = rc.gated_norm(c["h"], c["x"], gate=c["gate"], post_weight=c["post_weight"], spans=SPANS, want_y=False)
        ref, size = _residual(c, 1.0, False, 1e-6)
        inside("h alone", gh, ref, U * ref.abs() + F * size)
        assert none is None


def test_norm_in_place_and_row_counts():
    for N in (1, 2, 3, 4, 5, 63, 64, 65, 1000):
        c = _norm_case(2, [(N, 0)], 256, seed=N)
        gh, gy = _check_norm(c, "layer")
        out, y = rc.gated_norm(**c, h_out=c["h"])
        assert out is c["h"] and torch.equal(out, gh) and torch.equal(y, gy)


def test_norm_of_constant_and_large_rows():
    c = _norm_case(1, [(4, 0)], 512, seed=3, branch=False, mod=False)
    c["h"][:, 0] = 0.0
    c["h"][:, 1] = 3.0
    _, y = rc.gated_norm(**c, norm="layer")
    assert torch.equal(y[:, :2], torch.zeros_like(y[:, :2]))  # nothing but the mean
    c["h"] = c["h"] * 1e15
    _check_norm(c, "rms")
    c["h"] = (c["h"].float() * 1e-30).to(BF16)
    _check_norm(c, "layer")


def _check_norm_backward(c, kind, seed, rs=1.0, post_norm=False, eps=1e-6, with_dy=True, with_dh=True):
    shape = c["h"].shape
    dy = draw(shape, seed, 11) if with_dy else None
    dh = draw(shape, seed, 12) if with_dh else None
    got = rc.gated_norm_backward(dy, dh=dh, norm=kind, residual_scale=rs, post_norm=post_norm, eps=eps, **c)
    spans, post = c["spans"], post_norm or c["post_weight"] is not None
    h = c["h"].double()
    G = 1 + max(g for _, g in spans)
    if c["gate"] is not None or c["scale"] is not None:
        G = (c["gate"] if c["gate"] is not None else c["scale"]).shape[1]
    pick = torch.nn.functional.one_hot(torch.repeat_interleave(
        torch.tensor([g for _, g in spans]), torch.tensor([n for n, _ in spans])), G).double().t().to(DEV)
    grad, size = torch.zeros_like(h), torch.zeros_like(h)
    if with_dy:
        n, r = _n(h, kind, eps)
        w = 1.0 if c["weight"] is None else c["weight"].double()
        s = 1.0 if c["scale"] is None else 1 + _of(c["scale"], spans)
        Y = dy.double()
        dn = Y * s * w
        out = dn - n * (dn * n).mean(-1, keepdim=True)
        grad = r * (out - dn.mean(-1, keepdim=True) if kind == "layer" else out)
        # the mean's rounding reaches n as 2^-16 of r |h|
        off = n.abs() + r * (h.abs() + h.abs().mean(-1, keepdim=True))
        size = r * (dn.abs() + dn.abs().mean(-1, keepdim=True) + off * (dn.abs() * off).mean(-1, keepdim=True))
        if c["shift"] is not None:
            inside("dshift", got.shift, pick @ Y, F * (pick @ Y.abs()))
        if c["scale"] is not None:
            inside("dscale", got.scale, pick @ (Y * n * w), F * (pick @ (Y * off * w).abs()))
        if c["weight"] is not None:
            inside("dweight", got.weight, (Y * s * n).sum((0, 1)), F * (Y * s * off).abs().sum((0, 1)))
    if with_dh:
        grad, size = grad + dh.double(), size + dh.double().abs()
    inside("dh", got.h, grad, U * grad.abs() + F * size)
    if c["x"] is None:
        assert got.x is None and got.gate is None
        return dy, dh, got
    x, g = c["x"].double(), _of(c["gate"], spans)
    du, dsz = rs * grad * (1.0 if g is None else g), abs(rs) * size * (1.0 if g is None else g.abs())
    u, wp = x, 1.0 if c["post_weight"] is None else c["post_weight"].double()
    if post:
        xn = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
        rx = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
        if c["post_weight"] is not None:
            inside("dpost_weight", got.post_weight, (du * xn).sum((0, 1)), F * (dsz * xn.abs()).sum((0, 1)))
        u = xn * wp
        du, dsz = du * wp, dsz * abs(wp)
        dx = rx * (du - xn * (du * xn).mean(-1, keepdim=True))
        xsz = rx * (dsz + xn.abs() * (dsz * xn.abs()).mean(-1, keepdim=True))
    else:
        dx, xsz = du, dsz
    inside("dx", got.x, dx, U * dx.abs() + F * xsz)
    if c["gate"] is not None:
        inside("dgate", got.gate, pick @ (rs * grad * u), F * (pick @ (abs(rs) * size * u.abs())))
    return dy, dh, got


@pytest.mark.parametrize("C", [8, 64, 512, 520, 1024, 1152, 1928, 2560, 3080, 4096, 4104, 8192, 8200, 16384])
def test_norm_gradient_of_widths(C):
    _check_norm_backward(_norm_case(2, SPANS, C, seed=C), "layer", seed=C)
    _check_norm_backward(_norm_case(1, [(5, 0)], C, seed=C + 1, weight=True, post=True), "rms", seed=C, rs=0.5)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("parts", [dict(branch=False), dict(gate=False), dict(mod=False), dict(post=True),
                                   dict(weight=True, post=True), dict(weight=True, mod=False, gate=False)],
                         ids=lambda p: "-".join(p))
def test_norm_gradient_parts(parts, kind):
    c = _norm_case(2, SPANS, 640, seed=22, ld=24, **parts)
    _check_norm_backward(c, kind, seed=1, rs=0.7, eps=1e-5)
    _check_norm_backward(c, kind, seed=2, with_dh=False)
    if c["x"] is not None:
        _check_norm_backward(c, kind, seed=3, post_norm=True)
        c.update(scale=None, shift=None, weight=None)
        _check_norm_backward(c, kind, seed=4, with_dy=False)


@pytest.mark.parametrize("spans", [[(1, 0)], [(9, 1), (2, 0)], [(700, 0), (1, 1), (1500, 0), (333, 1), (3, 3)]],
                         ids=["one", "few", "many"])
def test_norm_gradient_of_spans(spans):
    c = _norm_case(2, spans, 1152, seed=31, weight=True, post=True)
    dy, dh, got = _check_norm_backward(c, "layer", seed=5)
    for g in range(c["scale"].shape[1]):
        if g not in [k for _, k in spans]:
            assert (got.scale[:, g] == 0).all() and (got.gate[:, g] == 0).all() and (got.shift[:, g] == 0).all()
    ws = torch.full((1 << 22,), float("nan"), device=DEV)
    again = rc.gated_norm_backward(dy, dh=dh, norm="layer", workspace=ws, **c)
    for a, b in zip(again, got):
        assert torch.equal(a, b)
    out = rc.gated_norm_backward(dy, dh=dh, norm="layer", dh_out=dh, dx=c["x"], **c)
    assert out.h is dh and out.x is c["x"]
    for a, b in zip(out, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("C", [64, 1024, 4096])
def test_norm_gradient_of_idle_row_groups(C):
    """The last rows of a chunk leave row groups idle: they add nothing, with
    eps = 0, and in place where a row's gradient overflows bf16."""
    for N in (1, 9, 13, 70):
        c = _norm_case(1, [(N, 0)], C, seed=N, post=True)
        _check_norm_backward(c, "rms", seed=N, post_norm=True, eps=0.0)
    h, dy = torch.ones(1, 9, C, dtype=BF16, device="cuda"), torch.zeros(1, 9, C, dtype=BF16, device="cuda")
    h[:, 8, 0] = 2.0
    dy[:, 8, 1] = 2.0 ** 127
    shift = torch.zeros(1, 1, C, dtype=BF16, device="cuda")
    g = rc.gated_norm_backward(dy, h * 2.0 ** -20, shift=shift, norm="rms", eps=0.0, dh_out=dy)
    assert g.h is dy and bool(torch.isinf(dy[0, 8, 1])) and float(dy[:, :8].abs().max()) == 0.0
    assert float(g.shift[0, 0, 1]) == 2.0 ** 127 and float(g.shift.abs().sum()) == 2.0 ** 127


def test_norm_gradient_against_differences():
    c = _norm_case(1, [(3, 0), (2, 1)], 64, seed=41, weight=True, post=True)
    dy, dh = draw(c["h"].shape, 41, 11), draw(c["h"].shape, 41, 12)
    got = rc.gated_norm_backward(dy, dh=dh, residual_scale=0.6, **c)

    def value(v):
        # h' at the given rows: its input differs by a constant
        u = v["x"] * torch.rsqrt(v["x"].square().mean(-1, keepdim=True) + 1e-6) * v["post_weight"]
        at = lambda m: m[:, [0, 0, 0, 1, 1]]  # noqa: E731
        u0 = base["x"] * torch.rsqrt(base["x"].square().mean(-1, keepdim=True) + 1e-6) * base["post_weight"]
        h = v["h"] + 0.6 * (at(v["gate"]) * u - at(base["gate"]) * u0)
        n, _ = _n(h, "layer", 1e-6)
        y = n * v["weight"] * (1 + at(v["scale"])) + at(v["shift"])
        return (y * dy.double()).sum() + (h * dh.double()).sum()

    base = {k: _d(t) for k, t in c.items() if k != "spans"}
    g = torch.Generator().manual_seed(3)
    for _ in range(3):
        step = {k: torch.randn(t.shape, generator=g, dtype=torch.float64).to(DEV) for k, t in base.items()}
        e = 1e-5
        diff = (value({k: t + e * step[k] for k, t in base.items()})
                - value({k: t - e * step[k] for k, t in base.items()})) / (2 * e)
        terms = [(got._asdict()[k].double() * step[k]) for k in base]
        along, scale = sum(t.sum() for t in terms), sum(t.norm() for t in terms)
        assert abs((along - diff).item()) <= 4 * U * scale.item()


def test_norm_of_no_rows():
    h = torch.empty(2, 0, 64, dtype=BF16, device=DEV)
    mod = torch.zeros(2, 1, 64, dtype=BF16, device=DEV)
    out, y = rc.gated_norm(h, h, gate=mod, scale=mod, shift=mod)
    assert out.shape == h.shape and y.shape == h.shape
    got = rc.gated_norm_backward(h, h, h, gate=mod, scale=mod, shift=mod)
    assert (got.gate == 0).all() and (got.scale == 0).all() and (got.shift == 0).all()


# ---------------------------------------------------------------- streams and graphs
def test_layer_operators_captured_and_on_a_stream():
    R, q, k, pos, wq, wk, _ = _rotary_case(128, (16, 56, 56), True, False, 1, 50, 4, seed=51)
    c = _norm_case(1, SPANS, 512, seed=52, post=True, weight=True)
    dq, dk, dy, dh = draw(q.shape, 51, 8), draw(q.shape, 51, 9), draw(c["h"].shape, 52, 11), draw(c["h"].shape, 52, 12)

    def run(stream=None):
        a = rc.qk_rotary(R, q, k, pos, q_norm=wq, k_norm=wk, stream=stream)
        b = rc.qk_rotary_backward(R, dq, dk, pos, q=q, k=k, q_norm=wq, k_norm=wk, stream=stream)
        d = rc.gated_norm(**c, stream=stream)
        e = rc.gated_norm_backward(dy, dh=dh, stream=stream, **c)
        return [*a, *b, *d, *e]

    ref = run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = run(s)
    s.synchronize()
    for a, b in zip(out, ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = run()
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, ref):
            assert torch.equal(a, b)
        run()
