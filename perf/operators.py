"""The gated linear recurrence and the input projection with 4-bit weights, as cases that can be timed.

Four families, each with cases from single tokens to the largest that a user of this package has:

  scan      h_t = f_t h_{t-1} + i_t v_t over whole sequences (`gated_forward`), alone (a prompt, a token) or
            followed by its adjoint (`gated_backward`: a training step)
  quantise  weights of an input projection to 4 bits with a scale per group (`quantize_projection`)
  project   u = B x + b with such weights (`input_projection_q4`)
  step      one token of a gated layer: projection and recurrence in one call (`gated_layer_step`)

`run` computes them with elementary torch operations in 32 bits, or with the package's kernels where `own` is true.
`exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

#: true: the calls that a user makes of the package's operators; false: elementary torch operations
own = False

_LARGEST = 1 << 27                             # most timesteps x channels of a drawn recurrence


def listed():
    fp32, bf16 = "fp32", "bf16"
    return [
        # generation with an unquantised projection: the next timestep of 32 sequences, where latency is all there is
        dict(name="scan-token", family="scan", dtype=bf16, B=32, L=1, H=1024, G=2, h0=True, ragged=False, backward=False),
        # three prompts of different lengths in one batch, rows at odd addresses
        dict(name="scan-prompts", family="scan", dtype=bf16, B=3, L=1531, H=1001, G=3, h0=True, ragged=True, backward=False),
        # training in fp32: the sizes of benchmark configuration 2
        dict(name="scan-train-fp32", family="scan", dtype=fp32, B=16, L=4096, H=1024, G=2, h0=False, ragged=False, backward=True),
        # training in bf16 with gates of its own for the input: the sizes of benchmark configuration 3
        dict(name="scan-train-bf16", family="scan", dtype=bf16, B=8, L=2048, H=2048, G=3, h0=False, ragged=False, backward=True),
        # training on long sequences: the sizes of benchmark configuration 5, the largest
        dict(name="scan-train-long", family="scan", dtype=bf16, B=4, L=65536, H=4096, G=2, h0=True, ragged=False, backward=True),
        # a small padded fine-tuning batch, ragged in every size
        dict(name="scan-train-padded", family="scan", dtype=fp32, B=5, L=777, H=333, G=3, h0=True, ragged=True, backward=True),
        # a trained layer of full matrices made ready for serving
        dict(name="quantise-full", family="quantise", H=4096, heads=1, G=2, group=64),
        # a small layer of narrow heads
        dict(name="quantise-heads", family="quantise", H=448, heads=7, G=3, group=32),
        # the next token of five sequences for a nonlinear cell of three gates, fp32 storage
        dict(name="project-token", family="project", dtype=fp32, B=5, L=1, H=1536, heads=4, G=3, group=128),
        # two prompts of no round length: rows enough that the products bound it
        dict(name="project-prompt", family="project", dtype=bf16, B=2, L=1999, H=2048, heads=1, G=2, group=64),
        # the next token of one sequence, full matrices: the weights are read once
        dict(name="step-one", family="step", dtype=bf16, B=1, H=4096, heads=1, G=2, group=64),
        # the next token of a batch, narrower heads and more gates
        dict(name="step-batch", family="step", dtype=bf16, B=48, H=2048, heads=4, G=3, group=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the family by its share of use, sizes over the logarithm of their ranges."""
    x = rng.random()
    if x < 0.55:
        H, B = _log(rng, 8, 4096), _log(rng, 1, 64)
        if rng.random() < 0.5:
            H = max(8, H // 8 * 8)             # model widths are multiples of eight more often than not
        L = 1 if rng.random() < 0.1 else _log(rng, 2, min(65536, max(32, _LARGEST // (B * H))))
        return dict(family="scan", dtype=rng.choice(("bf16", "fp32")), B=B, L=L, H=H, G=rng.choice((2, 3)),
                    h0=L == 1 or rng.random() < 0.5, ragged=L > 1 and rng.random() < 0.4,
                    backward=L > 1 and rng.random() < 0.6)
    heads, dh = rng.choice((1, 2, 3, 4, 8)), 64 * _log(rng, 1, 16)
    group = rng.choice([g for g in (32, 64, 128) if dh % g == 0])
    case = dict(H=heads * dh, heads=heads, group=group)
    if x < 0.65:
        return dict(case, family="quantise", G=rng.randint(1, 4))
    if x < 0.82:
        B = _log(rng, 1, 64)
        L = 1 if rng.random() < 0.5 else _log(rng, 1, max(1, 4096 // B))
        return dict(case, family="project", dtype=rng.choice(("bf16", "bf16", "fp32")), B=B, L=L, G=rng.randint(1, 4))
    return dict(case, family="step", dtype=rng.choice(("bf16", "bf16", "fp32")), B=_log(rng, 1, 64), G=rng.choice((2, 3)))


def _storage(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _weights(case, gen):
    dh = case["H"] // case["heads"]
    return torch.randn(case["G"], case["H"], dh, generator=gen, device="cuda") * dh ** -0.5


def _codes(W, group):
    """Codes -7 .. 7 (int8, W's shape) and bf16 scales [G][H][dh / group] of the nearest values on each group's grid: the
    scale is the group's largest magnitude / 7 in bf16, ties go to the even code.  Quotients in 64 bits, where no rounding
    of theirs can cross the middle between two codes."""
    w = W.view(*W.shape[:2], -1, group)
    scale = (w.abs().amax(-1).double() / 7).to(torch.bfloat16)
    s = scale.double().unsqueeze(-1)
    q = torch.where(s > 0, w.double() / s.clamp_min(1e-300), 0.0).round_().clamp_(-7, 7)
    return q.to(torch.int8).view(W.shape), scale


def prepare(case, seed):
    gen = _generator(seed)

    def normal(*shape, dtype, mean=0.0, std=1.0):
        t = torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)
        if std != 1.0:
            t.mul_(std)
        return t.add_(mean) if mean else t

    s = dict(case)
    f32 = torch.float32
    B, H, G = case.get("B"), case["H"], case["G"]
    if case["family"] == "scan":
        dt, L = _storage(case), case["L"]
        s["u"] = normal(B, L, G, H, dtype=dt)
        s["u"][:, :, 0] += 1.5                 # gates that remember for a few steps to a few hundred
        s["state"] = normal(B, H, dtype=f32, std=0.5) if case["h0"] else None
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            s["lengths"][0] = L
        if case["backward"]:
            s["g"] = normal(B, L, H, dtype=dt)
            s["dlast"] = normal(B, H, dtype=f32)
        return s
    W = _weights(case, gen)
    if case["family"] == "quantise":
        s["Wx"] = W
        return s
    s["codes"], s["scales"] = _codes(W, case["group"])
    s["bias"] = normal(G, H, dtype=f32, std=0.5)
    if case["family"] == "project":
        s["x"] = normal(B, case["L"], H, dtype=_storage(case))
    else:
        s["x"] = normal(B, H, dtype=_storage(case))
        s["bias"][0] += 1.5
        s["state"] = normal(B, H, dtype=f32, std=0.5)
    if own:
        import paper_2510_21450_amd as P
        s["Wq"] = P.pack_projection(s["codes"], s["scales"], n_heads=case["heads"])
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2510_21450_amd as P
    if s["family"] == "scan":
        h, last, ckpt = P.gated_forward(s["u"], s["state"], lengths=s["lengths"], checkpoints=s["backward"])
        out = {"h": h, "last": last}
        if s["backward"]:
            out["du"], out["dstate"] = P.gated_backward(s["u"], ckpt, s["g"], s["dlast"], lengths=s["lengths"])
        return out
    if s["family"] == "quantise":
        return {"W": P.dequantize_projection(P.quantize_projection(s["Wx"], n_heads=s["heads"], group=s["group"]))}
    if s["family"] == "project":
        return {"u": P.input_projection_q4(s["x"], s["Wq"], s["bias"])}
    y, state = P.gated_layer_step(s["x"], s["Wq"], s["state"], s["bias"])
    return {"y": y, "state": state}


# ---------------------------------------------------------------- plain forms, 32 bits
def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from zero, by doubling; a and b are overwritten, h is returned in b."""
    d, L = 1, a.shape[1]
    while d < L:
        b[:, d:] += a[:, d:] * b[:, :-d]
        if 2 * d < L:
            a[:, d:] = a[:, d:] * a[:, :-d]
        d *= 2
    return b


def _gates(s, u):
    """f, i, v in 32 bits"""
    u = u.float()
    f = torch.sigmoid(u[..., 0, :])
    i = torch.sigmoid(-u[..., 0, :]) if s["G"] == 2 else torch.sigmoid(u[..., 1, :])
    return f, i, u[..., -1, :]


def _run_plain(s):
    if s["family"] == "scan":
        return _scan_plain(s)
    if s["family"] == "quantise":
        q, scale = _codes(s["Wx"], s["group"])
        return {"W": _values(q, scale, s["group"])}
    W = _values(s["codes"], s["scales"], s["group"])
    u = _project_plain(s["x"].float(), W, s["heads"]) + s["bias"]
    if s["family"] == "project":
        return {"u": u.to(s["x"].dtype)}
    f, i, v = _gates(s, u)
    state = f * s["state"] + i * v
    return {"y": state.to(s["x"].dtype), "state": state}


def _values(codes, scales, group):
    w = codes.view(*codes.shape[:2], -1, group).float() * scales.float().unsqueeze(-1)
    return w.view(codes.shape)


def _project_plain(x, W, heads):
    """u[..., g, h] = sum_j W[g, h, j] x[..., head(h) dh + j], one product per head"""
    G, H, dh = W.shape
    rows = x.reshape(-1, H)
    u = torch.empty(rows.shape[0], G, H, device=x.device, dtype=x.dtype)
    for k in range(heads):
        at = slice(k * dh, (k + 1) * dh)
        u[:, :, at] = (rows[:, at] @ W[:, at].reshape(G * dh, dh).t()).view(-1, G, dh)
    return u.view(*x.shape[:-1], G, H)


def _scan_plain(s):
    dt, L = s["u"].dtype, s["u"].shape[1]
    f, i, v = _gates(s, s["u"])
    b = i * v
    valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(L, device=f.device) < s["lengths"][:, None]).unsqueeze(-1)
        f, b = torch.where(valid, f, 1.0), torch.where(valid, b, 0.0)
    if s["state"] is not None:
        b[:, 0] += f[:, 0] * s["state"]
    h = _scan(f.clone() if s["backward"] else f, b)
    last = h[:, -1].clone()
    out = {"h": (h if valid is None else torch.where(valid, h, 0.0)).to(dt), "last": last}
    if not s["backward"]:
        return out
    # mu_t = f_t (g_t + mu_{t+1}), the gradient of h_{t-1}; lambda_t = g_t + mu_{t+1}, that of h_t
    g = s["g"].to(torch.float32, copy=True)         # becomes lambda in place
    if valid is not None:
        g = torch.where(valid, g, 0.0)
    m = (f * g).flip(1)
    m[:, 0] += f[:, -1] * s["dlast"]
    m = _scan(f.flip(1), m).flip(1)
    out["dstate"] = m[:, 0].clone()
    lam = g
    lam[:, :-1] += m[:, 1:]
    lam[:, -1] += s["dlast"]
    del m
    before = torch.empty_like(h)
    before[:, 1:] = h[:, :-1]
    before[:, 0] = 0.0 if s["state"] is None else s["state"]
    del h
    du = torch.empty_like(s["u"])
    slope = torch.sigmoid(-s["u"][:, :, 0].float()) * torch.sigmoid(s["u"][:, :, 0].float())
    if s["G"] == 2:
        du[:, :, 0] = (lam * (before - v) * slope).to(dt)
    else:
        du[:, :, 0] = (lam * before * slope).to(dt)
        du[:, :, 1] = (lam * v * i * torch.sigmoid(-s["u"][:, :, 1].float())).to(dt)
    du[:, :, -1] = (lam * i).to(dt)
    if valid is not None:
        du *= valid.unsqueeze(-1)
    out["du"] = du
    return out


# ---------------------------------------------------------------- definitions, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["family"] == "scan":
        return _scan_exact(s)
    if case["family"] == "quantise":
        # nearest of the fifteen values of each group's grid, the even code where two are as near
        w = s["Wx"].double().view(case["G"], case["H"], -1, case["group"])
        unit = (w.abs().amax(-1, keepdim=True) / 7).to(torch.bfloat16).double()
        code = torch.floor(w / unit.clamp_min(1e-300))
        up = w - code * unit
        code += ((up > unit / 2) | ((up == unit / 2) & (code % 2 != 0))).double()
        return {"W": (code.clamp(-7, 7) * unit).reshape(s["Wx"].shape)}
    heads, dh, G = case["heads"], case["H"] // case["heads"], case["G"]
    W = s["codes"].double() * s["scales"].double().repeat_interleave(case["group"], -1)
    x = s["x"].double().view(-1, heads, dh).transpose(0, 1).contiguous()            # [heads][rows][dh]
    Wt = W.view(G, heads, dh, dh).permute(1, 3, 0, 2).reshape(heads, dh, G * dh)    # [heads][in][gate, out]
    u = torch.stack([x[k] @ Wt[k] for k in range(heads)]).view(heads, -1, G, dh)
    u = u.permute(1, 2, 0, 3).reshape(-1, G, case["H"]) + s["bias"].double()
    if case["family"] == "project":
        return {"u": u.view(case["B"], case["L"], G, case["H"])}
    keep = 1 / (1 + torch.exp(-u[:, 0]))
    enter = 1 / (1 + torch.exp(u[:, 0])) if G == 2 else 1 / (1 + torch.exp(-u[:, 1]))
    state = keep * s["state"].double() + enter * u[:, -1]
    return {"y": state, "state": state}


def _scan_exact(s):
    """The recurrence and its chain rule, a timestep after the other"""
    B, L, G, H = s["u"].shape
    at = [s["u"][:, :, k].transpose(0, 1).double() for k in range(G)]               # [L][B][H]
    keep = torch.sigmoid(at[0])
    enter = torch.sigmoid(-at[0]) if G == 2 else torch.sigmoid(at[1])
    add = enter * at[-1]
    live = torch.ones(L, B, 1, dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        live = (torch.arange(L, device="cuda")[:, None] < s["lengths"]).unsqueeze(-1)
        add.masked_fill_(~live, 0.0)
        keep.masked_fill_(~live, 1.0)
    h = torch.empty(L + 1, B, H, dtype=torch.float64, device="cuda")
    h[0] = 0.0 if s["state"] is None else s["state"].double()
    rows, fs, adds = h.unbind(0), keep.unbind(0), add.unbind(0)
    for t in range(L):
        torch.addcmul(adds[t], fs[t], rows[t], out=rows[t + 1])
    del add, adds
    out = {"h": (h[1:] if s["lengths"] is None else h[1:] * live).transpose(0, 1).clone(), "last": h[L].clone()}
    if not s["backward"]:
        return out
    # adj[t]: dL/dh_t with everything behind it, g_t + f_{t+1} adj[t+1]
    adj = s["g"].transpose(0, 1).double()
    if s["lengths"] is not None:
        adj.masked_fill_(~live, 0.0)
    adj = adj.contiguous()
    adj[L - 1] += s["dlast"].double()
    rows = adj.unbind(0)
    for t in range(L - 2, -1, -1):
        rows[t].addcmul_(fs[t + 1], rows[t + 1])
    out["dstate"] = keep[0] * adj[0]
    adj = torch.where(live, adj, 0.0)
    du = torch.empty(B, L, G, H, dtype=torch.float64, device="cuda")
    du[:, :, -1] = (adj * enter).transpose(0, 1)
    slope = keep * torch.sigmoid(-at[0])
    if G == 3:
        du[:, :, 0] = (adj * h[:-1] * slope).transpose(0, 1)
        du[:, :, 1] = (adj * at[2] * enter * torch.sigmoid(-at[1])).transpose(0, 1)
    else:
        du[:, :, 0] = (adj * (h[:-1] - at[1]) * slope).transpose(0, 1)
    out["du"] = du
    return out


def work(case):
    """Every input read once and every output written once.  Operations: per timestep and channel two for a step of the
    recurrence and about six for a gate, as much again twice for the adjoint; two for each weight and row of a product."""
    H, G = case["H"], case["G"]
    if case["family"] == "scan":
        B, L, esz = case["B"], case["L"], 2 if case["dtype"] == "bf16" else 4
        n = B * L * H
        ops = 3 + 6 * (G - 1)
        nbytes = n * esz * (G + 1) + 4 * B * H * (2 if case["h0"] else 1)
        if case["backward"]:
            nbytes += n * esz * (G + 1) + 2 * 4 * B * H
            ops += 2 * ops
        return {"bytes": nbytes, "flops": n * ops}
    weights = G * H * (H // case["heads"])
    if case["family"] == "quantise":
        return {"bytes": 8 * weights, "flops": 3 * weights}
    esz = 2 if case["dtype"] == "bf16" else 4
    nbytes = weights // 2 + 2 * weights // case["group"] + 4 * G * H
    rows = case["B"] * case.get("L", 1)
    if case["family"] == "project":
        nbytes += rows * H * esz * (1 + G)
    else:
        nbytes += rows * H * (2 * esz + 8)
    return {"bytes": nbytes, "flops": 2 * rows * weights}
