"""The gated linear recurrence (forward, adjoint, autograd) on the GPU against plain 64-bit forms on the CPU."""
import ctypes
import gc

import pytest
import torch

import gated_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2510_21450_amd as P
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return P


def problem(B, L, H, G, dtype, seed, h0=True, dlast=True):
    gen = torch.Generator().manual_seed(seed)
    u = torch.randn(B, L, G, H, generator=gen)
    u[:, :, 0] += 1.5
    if G == 3:
        u[:, :, 1] *= 2
    u = u.clamp(-ref.XMAX, ref.XMAX).to(dtype)
    g = torch.randn(B, L, H, generator=gen).to(dtype)
    s = torch.randn(B, H, generator=gen) if h0 else None
    d = torch.randn(B, H, generator=gen) if dlast else None
    return u, s, g, d


def cuda(t):
    return None if t is None else t.cuda()


def run_and_check(P, u, h0, g, dlast, lengths=None, device=None):
    """Both directions on the GPU; `device`: the tensors to use there, else copies."""
    du_, h0_, g_, dl_ = device if device is not None else (cuda(u), cuda(h0), cuda(g), cuda(dlast))
    n_ = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    h, last, ckpt = P.gated_forward(du_, h0_, lengths=n_, checkpoints=True)
    du, dh0 = P.gated_backward(du_, ckpt, g_, dl_, lengths=n_)
    torch.cuda.synchronize()
    w = ref.forward(u, h0, lengths)
    ref.check(h, w[0], w[2], "h")
    ref.check(last, w[1], w[3], "h_last")
    b = ref.backward(u, h0, g, dlast, lengths)
    ref.check(du, b[0], b[2], "dL_du")
    ref.check(dh0, b[1], b[3], "dL_dh0")
    return h, last, du, dh0


SIZES = [(1, 1, 1), (2, 1, 64), (3, 2, 7), (2, 16, 8), (2, 17, 65), (1, 127, 64), (1, 128, 72), (2, 129, 63), (1, 256, 8),
         (2, 257, 200), (3, 300, 96), (1, 1200, 16), (3, 513, 31), (2, 512, 64), (1, 513, 65), (2, 2100, 20), (1, 1025, 33), (9, 200, 460)]


@pytest.mark.parametrize("G", [2, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,L,H", SIZES)
def test_sizes(P, B, L, H, dtype, G):
    run_and_check(P, *problem(B, L, H, G, dtype, seed=B * 1000 + L + H))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h0,dlast", [(False, False), (True, False), (False, True)])
def test_states_that_are_not_given(P, dtype, h0, dlast):
    for L in (5, 200):
        run_and_check(P, *problem(2, L, 48, 2, dtype, seed=L, h0=h0, dlast=dlast))


@pytest.mark.parametrize("G", [2, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("L,lengths", [(9, [9, 0, 1, 8]), (300, [0, 300, 128, 129]), (300, [1, 127, 256, 257]), (140, [-5, 1000, 139, 12])])
def test_padded_batches(P, L, lengths, dtype, G):
    """Rows behind a sequence are not read (they hold NaN here), and are zeros in h and dL_du."""
    for H in (64, 33):
        u, h0, g, d = problem(4, L, H, G, dtype, seed=7 + L + H)
        for k, n in enumerate(ref.lengths_of(lengths, 4, L)):
            u[k, n:] = float("nan")
            g[k, n:] = float("nan")
        h, _, du, _ = run_and_check(P, u, h0, g, d, lengths)
        for k, n in enumerate(ref.lengths_of(lengths, 4, L)):
            assert (h[k, n:] == 0).all() and (du[k, n:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_address(P, dtype):
    """Tensors that start at an element's alignment only."""
    u, h0, g, d = problem(2, 150, 64, 2, dtype, seed=3)

    def odd(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        view = flat[1:].view(t.shape)
        view.copy_(t)
        return view
    run_and_check(P, u, h0, g, d, device=[odd(t) for t in (u, h0, g, d)])


@pytest.mark.parametrize("x", [-200.0, -88.0, 30.0, 200.0, float("inf"), float("-inf")])
def test_saturated_gates(P, x):
    """f = 0 and f = 1 to the last bit that matters, from either side."""
    u, h0, g, d = problem(1, 140, 16, 3, torch.float32, seed=11)
    u[:, :, 0, :8] = x
    u[:, :, 1, 4:] = x
    h, last, ckpt = P.gated_forward(u.cuda(), h0.cuda(), checkpoints=True)
    du, dh0 = P.gated_backward(u.cuda(), ckpt, g.cuda(), d.cuda())
    w, b = ref.forward(u, h0), ref.backward(u, h0, g, d)
    # the bound's GATE grows with |x|, but where a gate is saturated its error is below 2^-100 or 0
    for got, want, err in ((h, w[0], w[2]), (last, w[1], w[3]), (du, b[0], b[2]), (dh0, b[1], b[3])):
        got = got.double().cpu()
        assert torch.isfinite(got).all()
        assert ((got - want).abs() <= err + 2.0 ** -24 * want.abs() + 1e-30).all()


def test_tied_gate_keeps_small_inputs(P):
    """G = 2: i = 1 - f is formed without cancellation, so a memory that lets 1e-8 of the input in still gets it."""
    u = torch.zeros(1, 40, 2, 8)
    u[:, :, 0] = 18.0
    u[:, :, 1] = 1.0
    h, last, _ = P.gated_forward(u.cuda())
    want = ref.forward(u)[0]
    assert ((h.double().cpu() - want).abs() <= 64 * ref.EPS * want).all()


def test_nan_stays_where_it_belongs(P):
    """A NaN reaches the later states of its own channel, and the earlier gradients, nothing else."""
    u, h0, g, d = problem(2, 400, 24, 2, torch.float32, seed=5)
    u[1, 200, 1, 5] = float("nan")
    h, last, ckpt = P.gated_forward(u.cuda(), h0.cuda(), checkpoints=True)
    bad = torch.isnan(h).cpu()
    want = torch.zeros_like(bad)
    want[1, 200:, 5] = True
    assert torch.equal(bad, want) and torch.isnan(last).cpu().nonzero().tolist() == [[1, 5]]
    u, h0, g, d = problem(2, 400, 24, 2, torch.float32, seed=5)
    h, last, ckpt = P.gated_forward(u.cuda(), h0.cuda(), checkpoints=True)
    g[1, 200, 5] = float("nan")
    du, dh0 = P.gated_backward(u.cuda(), ckpt, g.cuda(), d.cuda())
    want = torch.zeros(2, 400, 2, 24, dtype=torch.bool)
    want[1, :201, :, 5] = True
    assert torch.equal(torch.isnan(du).cpu(), want) and torch.isnan(dh0).cpu().nonzero().tolist() == [[1, 5]]


def check_infinite(got, want, err, name):
    """Infinities where the 64-bit form has them, with its signs, and its values elsewhere."""
    got, far = got.double().cpu(), want.isinf()
    assert not want.isnan().any() and torch.equal(got[far], want[far]), f"{name}: infinities"
    half = ref.HALF_STEP[torch.bfloat16] if name.endswith("bf16") else ref.HALF_STEP[torch.float32]
    assert ((got - want).abs() <= err * (1 + half) + half * want.abs() + 1e-37)[~far].all(), name


@pytest.mark.parametrize("G", [2, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,L,H", [(2, 5, 24), (2, 30, 24), (2, 128, 24), (2, 300, 33), (1, 700, 24), (1, 2100, 16), (1, 1700, 40)])
def test_infinities_stay(P, B, L, H, dtype, G):
    """An infinite v, g or h0 is infinite from there on, as step by step: memories here fall below the least fp32 number within tens of steps,
    and a stretch's map must not turn an infinity into a NaN for it.  Other channels keep their values."""
    u, h0, g, d = problem(B, L, H, G, dtype, seed=L + H)
    u[:, :, 0] -= 4.5
    for k, x in enumerate((float("inf"), float("-inf"))):
        u[0, L // 3, -1, k] = x
        g[0, L // 2, 2 + k] = x
        h0[0, 4 + k] = x
        d[0, 6 + k] = x
    h, last, ckpt = P.gated_forward(u.cuda(), h0.cuda(), checkpoints=True)
    du, dh0 = P.gated_backward(u.cuda(), ckpt, g.cuda(), d.cuda())
    w, b = ref.forward(u, h0), ref.backward(u, h0, g, d)
    low = " bf16" if dtype == torch.bfloat16 else ""
    check_infinite(h, w[0], w[2], "h" + low)
    check_infinite(last, w[1], w[3], "h_last")
    check_infinite(du, b[0], b[2], "dL_du" + low)
    check_infinite(dh0, b[1], b[3], "dL_dh0")


@pytest.mark.parametrize("G", [2, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,L,H", [(1, 1500, 64), (2, 1300, 130), (1, 4500, 66), (1, 17500, 16), (1, 17000, 31)])
def test_looks_far_back(P, B, L, H, dtype, G):
    """Looks of 32 tiles by one and by two channels a thread, one and more trips of them, and of narrow tiles."""
    run_and_check(P, *problem(B, L, H, G, dtype, seed=B + L + H))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sequences_continue(P, dtype):
    """A sequence in pieces, the state updated in place, and token by token at its end: the states of the whole."""
    u, h0, _, _ = problem(2, 300, 40, 3, dtype, seed=21)
    want = ref.forward(u, h0)
    state = h0.cuda()
    h = torch.empty(2, 300, 40, dtype=dtype, device="cuda")
    at = 0
    for n in (140, 20, 129) + (1,) * 11:
        piece, last, _ = P.gated_forward(u[:, at:at + n].contiguous().cuda(), state, out=(torch.empty(2, n, 40, dtype=dtype, device="cuda"), state))
        assert last.data_ptr() == state.data_ptr()
        h[:, at:at + n] = piece
        at += n
    assert at == 300
    ref.check(h, want[0], want[2], "h")
    ref.check(state, want[1], want[3], "h_last")


def test_same_bits_every_time(P):
    """Many tiles in a chain and few chains: whom a tile finds ready differs between runs, the results do not."""
    u, h0, g, d = problem(2, 20000, 96, 2, torch.float32, seed=9)
    u, h0, g, d = cuda(u), cuda(h0), cuda(g), cuda(d)
    first = None
    for _ in range(4):
        h, last, ckpt = P.gated_forward(u, h0, checkpoints=True)
        got = (h, last, ckpt) + tuple(P.gated_backward(u, ckpt, g, d))
        if first is None:
            first = [t.clone() for t in got]
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def both(P, u, h0, g, d, **kw):
    h, last, ckpt = P.gated_forward(u, h0, checkpoints=True, **kw)
    return (h, last, ckpt) + tuple(P.gated_backward(u, ckpt, g, d, **kw))


def test_workspaces_of_any_content(P):
    """A workspace that holds anything, records of earlier calls among it, with and without the promise that nothing else writes to
    it; calls of different sizes and both directions on the same one."""
    cases = [[cuda(t) for t in problem(2, L, H, 2, torch.float32, seed=L)] for L, H in ((900, 130), (400, 64), (3000, 64))]
    want = [both(P, *c) for c in cases]
    size = max(P.gated_workspace_bytes(torch.float32, 2, c[0].shape[1], c[0].shape[3], 2) for c in cases)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    try:
        for reuse in (False, True):
            P.set_workspace_reuse(reuse)
            ws.random_(0, 256, generator=torch.Generator("cuda").manual_seed(1))
            if reuse:
                both(P, *cases[0], workspace=torch.empty_like(ws))       # another address: what is known of it is not known of ws
            for k in (0, 0, 1, 0, 2, 2, 1, 0):
                assert all(torch.equal(a, b) for a, b in zip(want[k], both(P, *cases[k], workspace=ws))), (reuse, k)
    finally:
        P.set_workspace_reuse(False)


def test_a_wait_that_runs_out(P):
    """One poll of a neighbour instead of millions: every workgroup still ends, what it did not get is NaN, and later calls on the same
    workspace are right again."""
    c = [cuda(t) for t in problem(1, 30000, 64, 2, torch.float32, seed=17)]
    want = both(P, *c)
    try:
        P.set_spin_limit(1)
        got = both(P, *c)
        torch.cuda.synchronize()
    finally:
        P.set_spin_limit(0)
    ok = (got[0] == want[0]) | torch.isnan(got[0])
    assert ok.all()
    again = both(P, *c)
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_what_a_wait_that_runs_out_leaves(P):
    """Every output of both directions is right or NaN, and some of each is NaN: 235 tiles that are on the device together and wait for one
    another look once."""
    u, h0, g, d = [cuda(t) for t in problem(1, 30000, 64, 2, torch.float32, seed=19)]
    h, last, ckpt = P.gated_forward(u, h0, checkpoints=True)
    want = P.gated_backward(u, ckpt, g, d)
    try:
        P.set_spin_limit(1)
        got = P.gated_forward(u, h0, checkpoints=True)
        back = P.gated_backward(u, ckpt, g, d)               # its waits alone: from right checkpoints
        from_bad = P.gated_backward(u, got[2], g, d)
        torch.cuda.synchronize()
    finally:
        P.set_spin_limit(0)
    pairs = list(zip(got, (h, last, ckpt))) + list(zip(back, want)) + list(zip(from_bad, want))
    for k, (a, b) in enumerate(pairs):
        assert ((a == b) | a.isnan()).all(), k
    assert got[0].isnan().any() and got[2].isnan().any() and back[0].isnan().any() and from_bad[0].isnan().any()
    # gradients of tiles whose checkpoint was not there need the state: not right by chance
    lost = got[2][0].isnan()
    assert from_bad[0][0, :, 0][lost[torch.arange(30000, device="cuda") // 128]].isnan().all()
    assert all(torch.equal(a, b) for a, b in zip(P.gated_backward(u, ckpt, g, d), want))


def scan_of_channels(u, h0):
    """64-bit states of a few channels of a long sequence on the GPU, by doubling."""
    f, i, v = ref.gates(u.double())
    a, b = f.clone(), i * v
    b[:, 0] += a[:, 0] * h0
    d = 1
    while d < a.shape[1]:
        b[:, d:] += a[:, d:] * b[:, :-d]
        a[:, d:] = a[:, d:] * a[:, :-d]
        d *= 2
    return b


def test_offsets_beyond_32_bits(P):
    """u of 4.8 GB in one sequence: the far rows are where they should be, in both directions."""
    B, L, H, G = 1, 145000, 4100, 2
    u = torch.empty(B, L, G, H, dtype=torch.float32, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    h0 = torch.ones(B, H, device="cuda")
    h, last, ckpt = P.gated_forward(u, h0, checkpoints=True)
    pick = [0, 1, 63, 64, 2049, 4099]
    want = scan_of_channels(u[..., pick], h0[:, pick])
    # memories are short here (f about 1/2): 40 half steps of the sum of magnitudes cover them
    assert ((h[..., pick].double() - want).abs() <= 40 * ref.EPS * (want.abs() + 4)).all()
    g = torch.zeros_like(h)
    g[:, -1] = 1.0
    g[:, L // 2] = 1.0
    du, dh0 = P.gated_backward(u, ckpt, g)
    f, i, v = ref.gates(u[..., pick].double())
    for t in (L - 1, L // 2):
        # what lies behind is forgotten in between: lam = 1
        assert ((du[:, t, 1][:, pick].double() - i[:, t]).abs() <= 40 * ref.EPS).all(), t
        slope = f[:, t] * (1 - f[:, t])
        before = scan_of_channels(u[:, t - 300:t][..., pick], torch.zeros(1, len(pick), device="cuda", dtype=torch.float64))[:, -1]
        assert ((du[:, t, 0][:, pick].double() - (before - v[:, t]) * slope).abs() <= 1e-5).all(), t
    assert (dh0.abs() < 1e-30).all()


def test_streams(P):
    """Calls on a stream of the caller's, and two at once on streams of their own."""
    cases = [problem(2, 3000, 128, 2, torch.float32, seed=k) for k in range(2)]
    want = []
    for u, h0, g, d in cases:
        h, last, ckpt = P.gated_forward(cuda(u), cuda(h0), checkpoints=True)
        want.append((h, last) + tuple(P.gated_backward(cuda(u), ckpt, cuda(g), cuda(d))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    data = [[cuda(t) for t in c] for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, (u, h0, g, d) in zip(streams, data):
            h, last, ckpt = P.gated_forward(u, h0, checkpoints=True, stream=s)
            got.append((h, last) + tuple(P.gated_backward(u, ckpt, g, d, stream=s)))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured(P):
    """Both directions in one graph, replayed on new inputs between eager calls."""
    u, h0, g, d = [cuda(t) for t in problem(3, 700, 72, 3, torch.bfloat16, seed=31)]
    n = torch.tensor([700, 300, 0], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h, last, ckpt = P.gated_forward(u, h0, lengths=n, checkpoints=True)
        P.gated_backward(u, ckpt, g, d, lengths=n)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, last, ckpt = P.gated_forward(u, h0, lengths=n, checkpoints=True)
        du, dh0 = P.gated_backward(u, ckpt, g, d, lengths=n)
    for k in range(4):
        new = problem(3, 700, 72, 3, torch.bfloat16, seed=40 + k)
        for t, s in zip((u, h0, g, d), new):
            t.copy_(s)
        n.copy_(torch.tensor([700 - k, 100 * k, 5], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        e_h, e_last, e_ckpt = P.gated_forward(u, h0, lengths=n, checkpoints=True)
        e_du, e_dh0 = P.gated_backward(u, e_ckpt, g, d, lengths=n)
        for a, b in ((h, e_h), (last, e_last), (du, e_du), (dh0, e_dh0)):
            assert torch.equal(a, b)


def kept(P):
    """Addresses of the workspaces whose records the library knows."""
    known = ctypes.CDLL(P.lib_path()).pararnn_workspace_known
    torch.cuda.synchronize()
    return {b["address"] for s in torch.cuda.memory_snapshot() for b in s["blocks"]
            if b["state"] == "active_allocated" and known(ctypes.c_void_p(b["address"]))}


def test_gated_calls_have_places_of_their_own(P):
    """More lengths than there are places do not push out what the solvers keep."""
    P.release_workspaces()
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    # (weights of which the solve is finite: equal bits say something)
    params = (torch.rand(2, 3, 260, generator=gen, device="cuda") * 2 - 1) * 0.9
    u, h0, g = rand(2, 2100, 3, 260), 0.1 * rand(2, 1, 260), rand(2, 2100, 1, 260)

    def solve():
        h = P.forward("gru_diag", params, u, h0, tol=1e-5, max_iter=16)[0]
        return (h, *P.backward("gru_diag", params, u, h0, h, g))
    want = solve()
    theirs = kept(P)
    assert theirs
    for tiles in range(2, 24):
        P.gated_forward(rand(2, tiles * 128, 2, 64))
    assert theirs <= kept(P) and 0 < len(kept(P) - theirs) <= 16
    assert all(torch.equal(a, b) for a, b in zip(want, solve()))
    P.release_workspaces()


def test_lengths_of_as_many_tiles_share_a_workspace(P):
    """Records depend on the tiles, not on the length: prompts that differ by a few steps use what the last one left."""
    P.release_workspaces()
    problems = [[cuda(t) for t in problem(2, L, 72, 2, torch.float32, seed=L)] for L in (1530, 1531, 1409, 1536)]
    want = [both(P, *c, workspace=torch.empty(P.gated_workspace_bytes(torch.float32, 2, c[0].shape[1], 72, 2), dtype=torch.uint8, device="cuda"))
            for c in problems]
    for k in (0, 1, 2, 3, 0):
        assert all(torch.equal(a, b) for a, b in zip(want[k], both(P, *problems[k]))), k
        assert len(kept(P)) == 1
    assert P.release_workspaces() == P.gated_workspace_bytes(torch.float32, 2, 1530, 72, 2)


# ---------------------------------------------------------------- autograd
@pytest.mark.parametrize("G", [2, 3])
def test_gradients_against_differences(P, G):
    """d loss / d u and d loss / d h0 against central differences of the 64-bit plain form."""
    u, h0, g, d = problem(2, 20, 3, G, torch.float32, seed=51)
    lengths = [20, 13]

    def loss(u, h0):
        h, last, _, _ = ref.forward(u, h0, lengths)
        return (h * g.double()).sum() + (last * d.double()).sum()
    ud, hd = u.double(), h0.double()
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    a, b = u.cuda().requires_grad_(), h0.cuda().requires_grad_()
    h, last = P.gated_apply(a, b, n)
    du, dh0 = torch.autograd.grad([h, last], [a, b], [g.cuda(), d.cuda()])
    step = 1e-5                          # differences are good to step^2 and 2^-53 / step: 1e-10
    gen = torch.Generator().manual_seed(1)
    for _ in range(12):
        at = int(torch.randint(0, ud.numel(), (1,), generator=gen))
        e = torch.zeros(ud.numel(), dtype=torch.float64)
        e[at] = step
        e = e.view_as(ud)
        want = float(loss(ud + e, hd) - loss(ud - e, hd)) / (2 * step)
        assert abs(float(du.flatten()[at]) - want) <= 2e-5 * max(1.0, abs(want))
    for at in range(hd.numel()):
        e = torch.zeros(hd.numel(), dtype=torch.float64)
        e[at] = step
        e = e.view_as(hd)
        want = float(loss(ud, hd + e) - loss(ud, hd - e)) / (2 * step)
        assert abs(float(dh0.flatten()[at]) - want) <= 2e-5 * max(1.0, abs(want))


def test_autograd_uses_what_there_is(P):
    """Only h, only h_last, expanded gradients, no gradient wanted, inputs without one."""
    u, h0, g, d = problem(2, 150, 16, 2, torch.float32, seed=61)
    for which in ("h", "last", "sum"):
        a, b = u.cuda().requires_grad_(), h0.cuda().requires_grad_()
        h, last = P.gated_apply(a, b)
        if which == "h":
            (h * g.cuda()).sum().backward()
            want = ref.backward(u, h0, g, None)
        elif which == "last":
            (last * d.cuda()).sum().backward()
            want = ref.backward(u, h0, None, d)
        else:
            h.sum().backward()
            want = ref.backward(u, h0, torch.ones_like(g), None)
        ref.check(a.grad, want[0], want[2], which)
        ref.check(b.grad, want[1], want[3], which)
    a = u.cuda().requires_grad_()
    h, _ = P.gated_apply(a, h0.cuda())
    h.sum().backward()
    assert a.grad is not None
    b = h0.cuda().requires_grad_()
    h, _ = P.gated_apply(u.cuda(), b)
    h.sum().backward()
    assert b.grad is not None
    with torch.no_grad():
        h, last = P.gated_apply(a, b)
    assert not h.requires_grad and not last.requires_grad


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("G", [2, 3])
def test_layer_is_its_parts(P, G, heads):
    """gated_layer against the calls it consists of, to the last bit."""
    gen = torch.Generator().manual_seed(71)
    B, L, H = 3, 200, 128
    x = torch.randn(B, L, H, generator=gen).to(torch.bfloat16).cuda().requires_grad_()
    W = (torch.randn(G, H, H // heads, generator=gen) * (H // heads) ** -0.5).cuda().requires_grad_()
    bias = torch.randn(G, H, generator=gen).cuda().requires_grad_()
    h0 = torch.randn(B, H, generator=gen).cuda().requires_grad_()
    n = torch.tensor([200, 0, 77], dtype=torch.int32, device="cuda")
    g, d = torch.randn(B, L, H, generator=gen).to(torch.bfloat16).cuda(), torch.randn(B, H, generator=gen).cuda()
    h, last = P.gated_layer(x, W, bias, h0, n, n_heads=heads)
    grads = torch.autograd.grad([h, last], [x, W, bias, h0], [g, d])
    u = P.input_projection(x.detach(), W.detach(), bias.detach(), n_heads=heads)
    e_h, e_last, ckpt = P.gated_forward(u, h0.detach(), lengths=n, checkpoints=True)
    du, dh0 = P.gated_backward(u, ckpt, g, d, lengths=n)
    dx, dW, db = P.input_projection_backward(x.detach(), W.detach(), du, n_heads=heads)
    for a, b in ((h, e_h), (last, e_last), (grads[0], dx), (grads[1], dW), (grads[2], db), (grads[3], dh0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("call", ["layer", "apply"])
def test_captured_training_step(P, call):
    """Forward and backward pass in one graph, replayed on new inputs.  While an eager graph of the same leaves lives the backward
    pass is refused (the engine would draw that graph's stream into the capture); afterwards it is captured."""
    gen = torch.Generator().manual_seed(81)
    x = torch.randn(2, 300, 64, generator=gen).to(torch.bfloat16).cuda().requires_grad_()
    W = (torch.randn(2, 64, 64, generator=gen) / 8).cuda().requires_grad_()
    u = torch.randn(2, 300, 2, 64, generator=gen).cuda().requires_grad_()
    h0 = torch.randn(2, 64, generator=gen).cuda().requires_grad_()
    g = torch.randn(2, 300, 64, generator=gen).cuda()
    leaves = (x, W, h0) if call == "layer" else (u, h0)
    g = g.to(torch.bfloat16) if call == "layer" else g

    def forward():
        return P.gated_layer(x, W, h0=h0)[0] if call == "layer" else P.gated_apply(u, h0)[0]

    def step():
        h = forward()
        return (h.detach(),) + torch.autograd.grad(h, leaves, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    alive = forward()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="eager graph"):
        with torch.cuda.graph(graph):
            step()
    del alive
    gc.collect()                        # the refused step's own graph, which the exception's frames hold
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        with torch.no_grad():
            for t in leaves:
                t.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


# ---------------------------------------------------------------- refusals
def test_refusals(P):
    u = torch.zeros(2, 10, 2, 16, device="cuda")
    h, last, ckpt = P.gated_forward(u, checkpoints=True)
    bad = [
        (ValueError, lambda: P.gated_forward(u.cpu())),
        (ValueError, lambda: P.gated_forward(u[0])),
        (ValueError, lambda: P.gated_forward(torch.zeros(2, 10, 4, 16, device="cuda"))),
        (ValueError, lambda: P.gated_forward(u.transpose(0, 1))),
        (KeyError, lambda: P.gated_forward(u.half())),
        (ValueError, lambda: P.gated_forward(u, torch.zeros(2, 16, device="cuda", dtype=torch.bfloat16))),
        (ValueError, lambda: P.gated_forward(u, torch.zeros(2, 16))),
        (ValueError, lambda: P.gated_forward(u, torch.zeros(1, 16, device="cuda"))),
        (ValueError, lambda: P.gated_forward(u, lengths=torch.zeros(2, device="cuda", dtype=torch.int64))),
        (ValueError, lambda: P.gated_forward(u, lengths=torch.zeros(3, device="cuda", dtype=torch.int32))),
        (ValueError, lambda: P.gated_forward(u, out=(h[:, :5], last))),
        (RuntimeError, lambda: P.gated_forward(torch.zeros(0, 10, 2, 16, device="cuda"))),
        (RuntimeError, lambda: P.gated_forward(torch.zeros(2, 0, 2, 16, device="cuda"))),
        (RuntimeError, lambda: P.gated_forward(torch.zeros(1, 3000, 2, 16, device="cuda"), workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
        (ValueError, lambda: P.gated_backward(u, ckpt[:, :, :8].contiguous(), h)),
        (ValueError, lambda: P.gated_backward(u, ckpt.double(), h)),
        (ValueError, lambda: P.gated_backward(u, ckpt, h[:, :5])),
        (ValueError, lambda: P.gated_backward(u, ckpt, h, torch.zeros(2, 15, device="cuda"))),
        (ValueError, lambda: P.gated_layer(torch.zeros(1, 3, 64, device="cuda"), torch.zeros(2, 64, 64))),
        (ValueError, lambda: P.gated_layer(torch.zeros(1, 3, 64, device="cuda"), torch.zeros(1, 64, 64, device="cuda"))),
        (ValueError, lambda: P.gated_layer(torch.zeros(1, 3, 64, device="cuda"), torch.zeros(2, 64, 64, device="cuda"), torch.zeros(2, 64))),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
    with pytest.raises(RuntimeError):           # H beyond what row offsets reach
        P.gated_forward(torch.zeros(1, 1, 2, (1 << 20) + 64, device="cuda"))


@pytest.mark.parametrize("call", ["layer", "apply"])
def test_second_derivatives_are_refused(P, call):
    """Gradients of a recorded backward pass have their values, and a derivative of them is an error, not a missing term."""
    u, h0, g, _ = problem(2, 70, 64, 2, torch.float32, seed=91)
    b = h0.cuda().requires_grad_()
    if call == "apply":
        a = u.cuda().requires_grad_()
        h, _ = P.gated_apply(a, b)
    else:
        a = u[:, :, 0].contiguous().cuda().requires_grad_()
        W = (torch.randn(2, 64, 64, generator=torch.Generator().manual_seed(92)) / 8).cuda()
        h, _ = P.gated_layer(a, W, None, b)
    want = torch.autograd.grad(h, (a, b), g.cuda(), retain_graph=True)
    got = torch.autograd.grad(h, (a, b), g.cuda(), create_graph=True)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(x.sum(), a, allow_unused=True)


@pytest.mark.parametrize("call", ["layer", "apply"])
@pytest.mark.parametrize("grad", [False, True])
def test_what_the_backward_pass_does_not_read_may_be_overwritten(P, call, grad):
    """A state buffer that takes the last state before the gradients are asked for, and a bias that an optimiser has stepped: the backward pass
    works from the checkpoints, and its gradients are the same to the last bit."""
    gen = torch.Generator().manual_seed(101)
    x = torch.randn(2, 300, 64, generator=gen).to(torch.bfloat16).cuda().requires_grad_()
    W = (torch.randn(2, 64, 64, generator=gen) / 8).cuda().requires_grad_()
    u = torch.randn(2, 300, 2, 64, generator=gen).cuda().requires_grad_()
    first, b = torch.randn(2, 64, generator=gen), torch.randn(2, 64, generator=gen)
    g = torch.randn(2, 300, 64, generator=gen).to(torch.bfloat16 if call == "layer" else torch.float32).cuda()
    got = []
    for overwrite in (False, True):
        state, bias = first.cuda().requires_grad_(grad), b.cuda().requires_grad_(grad)
        h, last = P.gated_layer(x, W, bias, state) if call == "layer" else P.gated_apply(u, state)
        if overwrite:
            with torch.no_grad():
                state.copy_(last)
                bias.mul_(0.5)
        leaves = ((x, W) if call == "layer" else (u,)) + ((state,) if grad else ()) + ((bias,) if grad and call == "layer" else ())
        got.append(torch.autograd.grad(h, leaves, g))
    assert all(torch.equal(p, q) for p, q in zip(*got))


def test_second_derivatives_by_way_of_the_state(P):
    """The gradients depend on the state in front and on the bias as well: a derivative of them with respect to those is an error too,
    also where they are results of other operations."""
    gen = torch.Generator().manual_seed(103)
    x = torch.randn(2, 70, 64, generator=gen).cuda()
    W = (torch.randn(2, 64, 64, generator=gen) / 8).cuda().requires_grad_()
    g = torch.randn(2, 70, 64, generator=gen).cuda()
    for leaf in (False, True):
        s, b = torch.randn(2, 64, generator=gen).cuda().requires_grad_(), torch.randn(2, 64, generator=gen).cuda().requires_grad_()
        h, _ = P.gated_layer(x, W, b if leaf else b * 2, s if leaf else s * 2)
        dW, = torch.autograd.grad(h, W, g, create_graph=True)
        for t in (s, b, W):
            with pytest.raises(RuntimeError, match="second derivatives"):
                torch.autograd.grad(dW.sum(), t, retain_graph=True)


def test_threads(P):
    """Calls of two threads on one stream and on two, kept workspaces and all."""
    import threading
    problems = [problem(3, 700, 96, 3, torch.bfloat16, seed=93 + k) for k in range(2)]
    on = [(u.cuda(), h0.cuda(), g.cuda()) for u, h0, g, _ in problems]

    def both(u, h0, g):
        h, last, ckpt = P.gated_forward(u, h0, checkpoints=True)
        return (h, last, *P.gated_backward(u, ckpt, g))

    want = [both(*t) for t in on]
    torch.cuda.synchronize()
    for streams in ((None, None), (torch.cuda.Stream(), torch.cuda.Stream())):
        got = [[], []]

        def work(k):
            with torch.cuda.stream(streams[k]):
                for _ in range(20):
                    got[k].append(both(*on[k]))

        threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        for k in range(2):
            assert len(got[k]) == 20
            for r in got[k]:
                for x, y in zip(r, want[k]):
                    assert torch.equal(x, y)
