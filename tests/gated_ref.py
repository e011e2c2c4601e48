"""Plain 64-bit forms of the gated linear recurrence and of 4-bit weights, on the CPU, with the bounds that the GPU tests
hold the kernels to (no kernel, nothing of the package).

Bounds.  A gate's value has a relative error of at most GATE half steps of fp32: the exponent's argument -x log2 e is rounded (its
half step times |x|, |x| <= XMAX in these tests), exp2 and the reciprocal are good to one step each (two half steps), the
sum and the products round.  A state is a sum of products of gates; each factor brings its own error, and joining the stretches of
a scan rounds at most three times more for a step.  So with |h|_t = f |h|_{t-1} + |i v| the error is at most err_t = f err_{t-1} +
(GATE + 3) 2^-24 |h|_t, and likewise against time for the adjoint."""
import torch

XMAX = 8.0
EPS = 2.0 ** -24
GATE = XMAX + 8
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def gates(u):
    f = torch.sigmoid(u[..., 0, :])
    i = torch.sigmoid(-u[..., 0, :]) if u.shape[-2] == 2 else torch.sigmoid(u[..., 1, :])
    return f, i, u[..., -1, :]


def lengths_of(lengths, B, L):
    return [L] * B if lengths is None else [min(max(int(n), 0), L) for n in lengths]


def forward(u, h0=None, lengths=None):
    """(h, last, err_h, err_last) in 64 bits; u [B][L][G][H], h0 [B][H] or None."""
    u = u.double()
    B, L, G, H = u.shape
    f, i, v = gates(u)
    b = i * v
    h, err = torch.zeros(B, L, H, dtype=torch.float64), torch.zeros(B, L, H, dtype=torch.float64)
    last, err_last = torch.zeros(B, H, dtype=torch.float64), torch.zeros(B, H, dtype=torch.float64)
    for k, n in enumerate(lengths_of(lengths, B, L)):
        x = torch.zeros(H, dtype=torch.float64) if h0 is None else h0[k].double()
        a, e = x.abs(), torch.zeros(H, dtype=torch.float64)
        for t in range(n):
            x = f[k, t] * x + b[k, t]
            a = f[k, t] * a + b[k, t].abs()
            e = f[k, t] * e + (GATE + 3) * EPS * a
            h[k, t], err[k, t] = x, e
        last[k], err_last[k] = x, e
    return h, last, err, err_last


def backward(u, h0, g, dlast, lengths=None):
    """(du, dh0, err_du, err_dh0) in 64 bits: the chain rule, a step after the other."""
    u = u.double()
    B, L, G, H = u.shape
    f, i, v = gates(u)
    om = torch.sigmoid(-u[..., 0, :])
    h, _, err_h, _ = forward(u, h0, lengths)
    du, err = torch.zeros_like(u), torch.zeros_like(u)
    dh0, err0 = torch.zeros(B, H, dtype=torch.float64), torch.zeros(B, H, dtype=torch.float64)
    zero = torch.zeros(H, dtype=torch.float64)
    for k, n in enumerate(lengths_of(lengths, B, L)):
        m = zero if dlast is None else dlast[k].double()
        a, e = m.abs(), zero
        for t in range(n - 1, -1, -1):
            gt = zero if g is None else g[k, t].double()
            lam, labs = gt + m, gt.abs() + a
            e = e + EPS * labs
            before = h[k, t - 1] if t else (zero if h0 is None else h0[k].double())
            eb = err_h[k, t - 1] if t else zero
            slope = f[k, t] * om[k, t]
            du[k, t, -1] = lam * i[k, t]
            err[k, t, -1] = i[k, t] * (e + (GATE + 2) * EPS * labs)
            at = before - v[k, t] if G == 2 else before
            mag = before.abs() + v[k, t].abs() if G == 2 else before.abs()
            du[k, t, 0] = lam * at * slope
            err[k, t, 0] = slope * (e * mag + labs * eb + (2 * GATE + 6) * EPS * labs * mag)
            if G == 3:
                si = i[k, t] * torch.sigmoid(-u[k, t, 1])
                du[k, t, 1] = lam * v[k, t] * si
                err[k, t, 1] = si * v[k, t].abs() * (e + (2 * GATE + 6) * EPS * labs)
            m, a = f[k, t] * lam, f[k, t] * labs
            e = f[k, t] * e + (GATE + 3) * EPS * a
        dh0[k], err0[k] = m, e
    return du, dh0, err, err0


def check(got, want, err, name):
    """|got - want| <= err and the rounding to got's type; got finite."""
    tol = err * (1 + HALF_STEP[got.dtype]) + HALF_STEP[got.dtype] * want.abs() + 1e-37
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    over = ((got - want).abs() - tol)
    worst = int(over.argmax())
    assert over.max() <= 0, (f"{name}: {got.flatten()[worst].item()} for {want.flatten()[worst].item()}, "
                             f"allowed {tol.flatten()[worst].item()}, at {worst} of {tuple(got.shape)}")


# ---------------------------------------------------------------- 4-bit weights
def quantise(W, group):
    """codes (int8) and scales (bf16 [G][H][dh / group]) by the definition, in 64 bits"""
    w = W.double().cpu().view(*W.shape[:2], -1, group)
    scale = (w.abs().amax(-1) / 7).to(torch.bfloat16)
    bad = ~torch.isfinite(w).all(-1)
    scale[bad] = float("nan")
    s = scale.double().unsqueeze(-1)
    q = torch.where(s > 0, w / torch.where(s > 0, s, 1.0), 0.0).round().clamp(-7, 7)
    return q.nan_to_num(0.0).to(torch.int8).view(W.shape), scale


def values(codes, scales):
    group = codes.shape[-1] // scales.shape[-1]
    return codes.double() * scales.double().repeat_interleave(group, -1)


def project(x, W, bias, heads):
    """(u, magnitude): sum_j W x and sum_j (|W| + 24 s-like terms) |x| are both linear in |x|; x [rows][H], W [G][H][dh]"""
    G, H, dh = W.shape
    xs = x.double().cpu().view(-1, heads, dh)
    Ws = W.view(G, heads, dh, dh)
    u = torch.stack([(xs[:, k] @ Ws[:, k].reshape(G * dh, dh).t()).view(-1, G, dh) for k in range(heads)], 2)
    u = u.reshape(-1, G, H)
    return u if bias is None else u + bias.double().cpu()
