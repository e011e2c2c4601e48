"""4-bit weights of the input projection, their products and the gated layer's single step on the GPU against plain 64-bit
forms on the CPU."""
import pytest
import torch

import gated_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2510_21450_amd as P
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return P


def weights(G, heads, dh, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(G, heads * dh, dh, generator=gen) * dh ** -0.5


def bound(x, W, scales, heads, rounded_weights=False):
    """Error of u from sums in fp32: the products with a code's 24 + q and the 24 taken out (together below 56 of scale s for
    each |x|), at most 64 + dh / 32 roundings of a running sum on the way; bf16 weights: half a step each."""
    G, H, dh = W.shape
    s = scales.double().repeat_interleave(dh // scales.shape[-1], -1)
    e = ref.project(x.double().abs(), s * 56 * (64 + dh / 32) * ref.EPS, None, heads)
    if rounded_weights:
        e = e + ref.project(x.double().abs(), W.abs() * 2.0 ** -8, None, heads)
    return e


# ---------------------------------------------------------------- quantising
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("G,heads,dh", [(1, 1, 128), (2, 3, 128), (3, 1, 256), (1, 2, 384)])
def test_nearest_values(P, G, heads, dh, group):
    W = weights(G, heads, dh, seed=dh + group)
    Wq = P.quantize_projection(W.cuda(), n_heads=heads, group=group)
    codes, scales = ref.quantise(W, group)
    assert (Wq.G, Wq.H, Wq.n_heads, Wq.group) == (G, heads * dh, heads, group)
    assert torch.equal(P.dequantize_projection(Wq).cpu().double(), ref.values(codes, scales))
    packed = P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads)
    assert torch.equal(packed.packed, Wq.packed)
    assert torch.equal(packed.scales.view(torch.int16), Wq.scales.view(torch.int16))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_values_at_the_borders(P, group):
    """Ties, one step beside them, groups of zeros, of subnormals, of one value, with an infinity, with a NaN; rows at a
    4-byte address."""
    W = torch.zeros(1, 128, 128)
    s = 0.0078125 * 1.25                                    # a bf16 number; 7 s is the largest of each group below
    mid = (torch.arange(32, dtype=torch.float32) % 7 + 0.5) * s
    W[0, 0:16] = mid.repeat(4)
    W[0, 16:32] = torch.nextafter(mid, torch.tensor(1e9)).repeat(4)
    W[0, 32:48] = torch.nextafter(mid, torch.tensor(-1e9)).repeat(4)
    W[0, 0:48, ::32] = 7 * s
    W[0, 8:48:2] *= -1
    W[0, 48] = 1e-41
    W[0, 49, 3] = 3.4e38
    W[0, 50, 5] = float("inf")
    W[0, 51, 127] = float("nan")
    W[0, 52, 64] = -2.5
    flat = torch.empty(W.numel() + 1, device="cuda")
    view = flat[1:].view(W.shape)
    view.copy_(W)
    got = P.dequantize_projection(P.quantize_projection(view, group=group)).cpu().double()
    codes, scales = ref.quantise(W, group)
    want = ref.values(codes, scales)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def test_codes_from_elsewhere(P):
    """All sixteen codes, and what lies outside them; negative and zero scales."""
    gen = torch.Generator().manual_seed(2)
    codes = torch.randint(-12, 12, (2, 128, 64), generator=gen, dtype=torch.int8)
    scales = torch.randn(2, 128, 2, generator=gen).to(torch.bfloat16)
    scales[0, 3, 1] = 0.0
    got = P.dequantize_projection(P.pack_projection(codes.cuda(), scales.cuda(), n_heads=2)).cpu().double()
    assert torch.equal(got, ref.values(codes.clamp(-8, 7), scales))


# ---------------------------------------------------------------- products
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,heads,dh,group", [(1, 1, 64, 32), (3, 3, 64, 64), (2, 2, 128, 128), (4, 1, 192, 64), (2, 1, 576, 32), (1, 2, 640, 128)])
@pytest.mark.parametrize("rows", [1, 5, 16, 17, 33, 64, 65, 130])
def test_products(P, rows, G, heads, dh, group, dtype):
    gen = torch.Generator().manual_seed(rows + dh)
    W = weights(G, heads, dh, seed=rows)
    codes, scales = ref.quantise(W, group)
    codes[0, 0, :8] = -8
    x = torch.randn(rows, heads * dh, generator=gen).to(dtype)
    bias = torch.randn(G, heads * dh, generator=gen) if rows % 2 else None
    Wq = P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads)
    B = 5 if rows % 5 == 0 else 1
    u = P.input_projection_q4(x.view(B, rows // B, -1).cuda(), Wq, None if bias is None else bias.cuda())
    V = ref.values(codes, scales)
    want = ref.project(x, V, bias, heads)
    many = dtype == torch.bfloat16 and rows > P.q4_exact_rows(heads * dh, G, heads)
    err = bound(x, V, scales, heads, rounded_weights=many) + 4 * ref.EPS * (0 if bias is None else bias.double().abs())
    ref.check(u.view(rows, G, -1), want, err, "u")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,heads,dh,group", [(8, 1, 2048, 128), (3, 1, 4096, 32), (8, 2, 1024, 64)])
@pytest.mark.parametrize("beyond", [0, 1, 300])
def test_products_of_many_rows(P, beyond, G, heads, dh, group, dtype):
    """At the border between the two ways for bf16, and behind it."""
    rows = P.q4_exact_rows(heads * dh, G, heads) + beyond
    assert 64 <= rows < 4000
    gen = torch.Generator().manual_seed(rows)
    codes, scales = ref.quantise(weights(G, heads, dh, seed=dh), group)
    x = torch.randn(rows, heads * dh, generator=gen).to(dtype)
    bias = torch.randn(G, heads * dh, generator=gen)
    Wq = P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads)
    u = P.input_projection_q4(x.view(1, rows, -1).cuda(), Wq, bias.cuda())
    V = ref.values(codes, scales)
    err = bound(x, V, scales, heads, rounded_weights=dtype == torch.bfloat16 and beyond > 0) + 4 * ref.EPS * bias.double().abs()
    ref.check(u.view(rows, G, -1), ref.project(x, V, bias, heads), err, "u")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,G,heads,dh,group", [(2100, 4, 3, 64, 64), (2049, 4, 3, 64, 32), (900, 4, 3, 192, 64), (900, 3, 5, 192, 32),
                                                   (1700, 3, 1, 576, 32), (1700, 3, 1, 640, 64), (1153, 8, 1, 512, 128), (1153, 8, 1, 512, 32)])
def test_products_in_tiles(P, rows, G, heads, dh, group, dtype):
    """Rows and channels that end inside a tile, one unit of inputs and odd numbers of them, sums of one wave and of two."""
    codes, scales = ref.quantise(weights(G, heads, dh, seed=rows), group)
    x = torch.randn(rows, heads * dh, generator=torch.Generator().manual_seed(rows)).to(dtype)
    bias = torch.randn(G, heads * dh, generator=torch.Generator().manual_seed(dh))
    Wq = P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads)
    flat = torch.full((rows * G * heads * dh + 2,), 5.0, dtype=dtype, device="cuda")
    u = P.input_projection_q4(x.view(1, rows, -1).cuda(), Wq, bias.cuda(), out=flat[1:-1].view(1, rows, G, heads * dh))
    V = ref.values(codes, scales)
    ref.check(u.view(rows, G, -1), ref.project(x, V, bias, heads), bound(x, V, scales, heads) + 4 * ref.EPS * bias.double().abs(), "u")
    assert flat[0] == 5 and flat[-1] == 5
    again = P.input_projection_q4(x.view(1, rows, -1).cuda(), Wq, bias.cuda())
    assert torch.equal(u, again)


def rounding_shows(G, dh, group, rows):
    """codes, scales, x and bias whose products cancel: inputs 1 and -7 under codes 7 and 1 take each other out exactly, and 7 s of the scale
    148 / 128 lies in the middle between two bf16 numbers: in bf16 each pair is off by 2^-5 of the inputs.  What is summed up are whole numbers
    below 2^24 (times a power of two), so that fp32 sums in any order are exact and u is the bias, rounded."""
    even = torch.arange(dh) % 2 == 0
    codes = torch.where(even, 7, 1).to(torch.int8).expand(G, dh, dh).contiguous()
    scales = torch.full((G, dh, dh // group), 148 / 128, dtype=torch.bfloat16)
    x = torch.where(even, 1.0, -7.0) * 2.0 ** (torch.arange(rows) % 3).unsqueeze(1)
    bias = torch.randn(G, dh, generator=torch.Generator().manual_seed(group))
    return codes, scales, x.to(torch.bfloat16), bias


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("G,dh,beyond", [(3, 1024, -64), (3, 1024, 1), (3, 1024, 2500), (8, 2048, 5)])
def test_any_number_of_rows_sees_the_weights(P, G, dh, beyond, group):
    """A prompt of many rows is multiplied with the same weights as the tokens after it: none of them is rounded."""
    rows = P.q4_exact_rows(dh, G, 1) + beyond
    codes, scales, x, bias = rounding_shows(G, dh, group, rows)
    Wq = P.pack_projection(codes.cuda(), scales.cuda())
    u = P.input_projection_q4(x[None].cuda(), Wq, bias.cuda())
    want = bias.to(torch.bfloat16).expand(1, rows, G, dh)
    assert torch.equal(u.cpu(), want)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_rounded_weights_where_they_are_asked_for(P, group):
    """set_q4_products(1): the weights rounded to bf16 from q4_exact_rows on, the codes up to there, and the codes again under 0."""
    G, dh = 3, 1024
    rows = P.q4_exact_rows(dh, G, 1)
    codes, scales, x, bias = rounding_shows(G, dh, group, rows + 7)
    Wq = P.pack_projection(codes.cuda(), scales.cuda())
    call = lambda n: P.input_projection_q4(x[None, :n].contiguous().cuda(), Wq, bias.cuda())
    exact = bias.to(torch.bfloat16)
    # 512 pairs that are 2^-5 off each, times 1, 2 or 4: whole multiples of 2^-7 below 2^24 of them, exact sums as well
    rounded = ref.project(x, ref.values(codes, scales).to(torch.bfloat16).double(), bias, 1)
    try:
        P.set_q4_products(1)
        assert torch.equal(call(rows)[0].cpu(), exact.expand(rows, G, dh))
        ref.check(call(rows + 7)[0], rounded, 4 * ref.EPS * rounded.abs(), "u")
    finally:
        P.set_q4_products(0)
    assert torch.equal(call(rows + 7)[0].cpu(), exact.expand(rows + 7, G, dh))
    for mode in (-1, 2):
        with pytest.raises(RuntimeError):
            P.set_q4_products(mode)


def low_bits(rows, G, heads, dh, group, seed):
    """fp32 inputs whose products cancel down to the last of their three bf16 terms.  Neighbours under the same code are a and -b with a, b of
    65792 + {0, 1}: the terms 65536, 256 and 0 or 1, the first two the same in both.  Sums of code times x are whole numbers below
    8 x 65793 x 16 < 2^24 for the 16 pairs of any 32 inputs, and those of all pairs below 8 dh / 2 < 2^24 once the pairs are whole, so fp32 sums
    in any order are exact; scales are powers of two.  Without the third terms u would be 0."""
    gen = torch.Generator().manual_seed(seed)
    H = heads * dh
    x = (65792.0 + torch.randint(0, 2, (rows, H), generator=gen)) * torch.tensor([1.0, -1.0]).repeat(H // 2)
    codes = torch.randint(-8, 8, (G, H, dh // 2), generator=gen, dtype=torch.int8).repeat_interleave(2, -1)
    scales = (2.0 ** torch.randint(-3, 3, (G, H, 1), generator=gen)).expand(G, H, dh // group).to(torch.bfloat16).contiguous()
    return x, codes, scales


def two_terms(x):
    upper = lambda t: (t.view(torch.int32) & -65536).view(torch.float32)
    return upper(x) + upper(x - upper(x))


@pytest.mark.parametrize("rows,G,heads,dh,group", [(1, 2, 1, 64, 32), (3, 3, 2, 128, 128), (16, 1, 1, 640, 64), (16, 3, 1, 4096, 64), (20, 2, 1, 192, 32),
                                                   (64, 4, 3, 192, 64), (2100, 4, 3, 64, 64), (900, 3, 5, 192, 32), (1153, 8, 1, 512, 128)])
def test_every_bit_of_fp32_inputs_counts(P, rows, G, heads, dh, group):
    x, codes, scales = low_bits(rows, G, heads, dh, group, seed=rows + dh)
    V = ref.values(codes, scales)
    want = ref.project(x, V, None, heads)
    assert (ref.project(two_terms(x), V, None, heads) == 0).all() and (want != 0).double().mean() > 0.8
    u = P.input_projection_q4(x[None].cuda(), P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads))
    assert torch.equal(u.view(rows, G, -1).double().cpu(), want)


@pytest.mark.parametrize("B,G,heads,dh,group", [(1, 2, 1, 256, 32), (5, 3, 2, 128, 128), (20, 2, 1, 640, 64), (64, 3, 1, 512, 64)])
def test_every_bit_of_fp32_inputs_counts_in_a_step(P, B, G, heads, dh, group):
    """v alone has codes that are not zero: f and i are sig(bias) and h' = f h + i v, to the gates' and three more roundings."""
    x, codes, scales = low_bits(B, G, heads, dh, group, seed=B + dh)
    codes[:-1] = 0
    H = heads * dh
    bias = torch.randn(G, H, generator=torch.Generator().manual_seed(B)).clamp(-ref.XMAX, ref.XMAX)
    bias[-1] = 0
    h = torch.randn(B, H, generator=torch.Generator().manual_seed(dh))
    f, i, v = ref.gates(ref.project(x, ref.values(codes, scales), bias, heads))
    mag = f * h.double().abs() + i * v.abs()
    y, nxt = P.gated_layer_step(x.cuda(), P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads), h.cuda(), bias.cuda())
    assert (v != 0).double().mean() > 0.8
    ref.check(nxt, f * h.double() + i * v, (ref.GATE + 3) * ref.EPS * mag, "h_next")
    assert torch.equal(y, nxt)


def test_products_with_the_codes_take_no_workspace(P):
    """Many rows of bf16 allocate their outputs and nothing else, unless the weights are to be rounded."""
    G, dh = 8, 2048
    Wq = P.quantize_projection(weights(G, 1, dh, seed=51).cuda())
    x = torch.randn(1, P.q4_exact_rows(dh, G, 1) + 1, dh, device="cuda").to(torch.bfloat16)

    def extra():
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        u = P.input_projection_q4(x, Wq)
        return torch.cuda.max_memory_allocated() - before - u.numel() * 2
    try:
        assert extra() < 1 << 20
        P.set_q4_products(1)
        assert extra() >= 2 * G * dh * dh
    finally:
        P.set_q4_products(0)


def test_a_row_keeps_to_itself(P):
    """A NaN in one row, an infinity in another, both in one head: those rows of that head alone, in tiles as in single rows."""
    Wq = P.quantize_projection(weights(4, 3, 64, seed=9).cuda(), n_heads=3)
    for rows in (3, 2100):
        for dtype in (torch.float32, torch.bfloat16):
            x = torch.randn(rows, 192, generator=torch.Generator().manual_seed(rows)).to(dtype).cuda()
            want = P.input_projection_q4(x[None], Wq)[0]
            x[1, 70], x[rows - 1, 3] = float("nan"), float("inf")
            u = P.input_projection_q4(x[None], Wq)[0]
            hit = torch.zeros(rows, 1, 192, dtype=torch.bool, device="cuda")
            hit[1, :, 64:128] = hit[rows - 1, :, :64] = True
            hit = hit.expand_as(u)
            assert not u[hit].isfinite().any() and torch.equal(u[~hit], want[~hit])


def test_one_row_of_another_batch_is_the_same(P):
    """A sequence's pre-activations do not depend on how many others there are beside it (bits, up to the exact rows)."""
    W = weights(3, 2, 256, seed=4).cuda()
    Wq = P.quantize_projection(W, n_heads=2, group=64)
    x = torch.randn(64, 1, 512, generator=torch.Generator().manual_seed(4)).cuda()
    alone = P.input_projection_q4(x[:1].contiguous(), Wq)
    for n in (2, 16):
        assert torch.equal(P.input_projection_q4(x[:n].contiguous(), Wq)[:1], alone)


def test_unaligned_outputs_and_rows_behind(P):
    """u at an element's alignment only, with guards around it that stay as they are."""
    Wq = P.quantize_projection(weights(2, 1, 128, seed=6).cuda(), group=32)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(3, 1, 128, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
        flat = torch.full((1 + 3 * 256 + 7,), 5.0, dtype=dtype, device="cuda")
        u = P.input_projection_q4(x, Wq, out=flat[1:1 + 3 * 256].view(3, 1, 2, 128))
        assert torch.equal(u, P.input_projection_q4(x, Wq))
        assert (flat[:1] == 5).all() and (flat[1 + 3 * 256:] == 5).all()


# ---------------------------------------------------------------- a token of a gated layer
def step_reference(x, V, scales, h, bias, heads, G):
    u = ref.project(x, V, bias, heads)
    e = bound(x, V, scales, heads) + 4 * ref.EPS * (0 if bias is None else bias.double().abs())
    f, i, v = ref.gates(u)
    s = torch.zeros_like(f) if h is None else h.double()
    want = f * s + i * v
    # the slope of either gate is at most 1/4; the gates themselves as in gated_ref, |u| may exceed XMAX by little
    mag = f * s.abs() + i * v.abs()
    err = 0.25 * e[:, 0] * s.abs() + i * e[:, -1] + 0.25 * (e[:, 0] if G == 2 else e[:, 1]) * v.abs() + (ref.GATE + 8) * ref.EPS * mag
    return want, err


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,heads,dh,group", [(2, 1, 64, 32), (3, 2, 64, 64), (2, 1, 640, 128), (3, 1, 512, 32)])
@pytest.mark.parametrize("B", [1, 3, 16, 20, 48, 64, 70, 129])
def test_step(P, B, G, heads, dh, group, dtype):
    gen = torch.Generator().manual_seed(B + dh)
    codes, scales = ref.quantise(weights(G, heads, dh, seed=B), group)
    x = torch.randn(B, heads * dh, generator=gen).to(dtype)
    bias = torch.randn(G, heads * dh, generator=gen) if B % 2 else None
    h = torch.randn(B, heads * dh, generator=gen) if B != 3 else None
    Wq = P.pack_projection(codes.cuda(), scales.cuda(), n_heads=heads)
    y, nxt = P.gated_layer_step(x.cuda(), Wq, None if h is None else h.cuda(), None if bias is None else bias.cuda())
    want, err = step_reference(x, ref.values(codes, scales), scales, h, bias, heads, G)
    ref.check(nxt, want, err, "h_next")
    ref.check(y, want, err, "y")
    assert torch.equal(y, nxt.to(dtype))
    if h is not None:                            # in place
        state = h.cuda()
        y2, n2 = P.gated_layer_step(x.cuda(), Wq, state, None if bias is None else bias.cuda(), out=(torch.empty_like(y), state))
        assert n2.data_ptr() == state.data_ptr() and torch.equal(n2, nxt) and torch.equal(y2, y)


def test_step_is_captured(P):
    Wq = P.quantize_projection(weights(2, 1, 256, seed=8).cuda())
    x, h = torch.randn(4, 256, device="cuda"), torch.randn(4, 256, device="cuda")
    y = torch.empty_like(x)
    P.gated_layer_step(x, Wq, h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.gated_layer_step(x, Wq, h, out=(y, h))
    for _ in range(4):
        before = h.clone()
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        e_y, e_h = P.gated_layer_step(x, Wq, before)
        assert torch.equal(y, e_y) and torch.equal(h, e_h)


@pytest.mark.parametrize("rows", [5, 200, 1700, -1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_are_captured(P, rows, dtype):
    """Replays on new inputs with eager calls between them and on another stream, for every way that the products take."""
    G, heads, dh = (3, 1, 640) if rows > 0 else (8, 1, 2048)
    rows = rows if rows > 0 else P.q4_exact_rows(dh, G, 1) + 5
    Wq = P.quantize_projection(weights(G, heads, dh, seed=21).cuda(), n_heads=heads)
    gen = torch.Generator(device="cuda").manual_seed(22)
    x = torch.randn(1, rows, dh, generator=gen, device="cuda").to(dtype)
    P.input_projection_q4(x, Wq)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u = P.input_projection_q4(x, Wq)
    side = torch.cuda.Stream()
    for _ in range(3):
        x.copy_(torch.randn(1, rows, dh, generator=gen, device="cuda"))
        graph.replay()
        want = P.input_projection_q4(x, Wq)
        assert torch.equal(u, want)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = P.input_projection_q4(x, Wq)
        raw = P.input_projection_q4(x, Wq, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(other, want) and torch.equal(raw, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_offsets_beyond_32_bits(P, dtype):
    """More than 2^31 outputs and 2^30 inputs: the last rows are what they are by themselves."""
    Wq = P.quantize_projection(weights(2, 64, 64, seed=31).cuda(), n_heads=64)
    x = torch.randn(1, 300000, 4096, device="cuda", generator=torch.Generator(device="cuda").manual_seed(32), dtype=dtype)
    u = P.input_projection_q4(x, Wq)
    assert u.numel() > 2 ** 31 and torch.equal(u[:, -5000:], P.input_projection_q4(x[:, -5000:], Wq))
    assert torch.equal(u[:, :5000], P.input_projection_q4(x[:, :5000], Wq))


# ---------------------------------------------------------------- together
def test_a_layer_from_training_to_serving(P):
    """A training step, the weights to 4 bits, a padded batch of prompts, then tokens: against the plain form of the 4-bit
    layer over whole sequences.  bf16; few rows, so that prompt and tokens see the same weights."""
    gen = torch.Generator().manual_seed(91)
    B, L, T, H, heads, G = 3, 20, 6, 256, 2, 3
    x = torch.randn(B, L + T, H, generator=gen).to(torch.bfloat16)
    W = weights(G, heads, H // heads, seed=91).cuda().requires_grad_()
    bias = torch.randn(G, H, generator=gen).cuda().requires_grad_()
    h, _ = P.gated_layer(x.cuda(), W, bias, n_heads=heads)
    gW, gb = torch.autograd.grad(h.float().square().mean(), (W, bias))
    W, bias = (W - 0.1 * gW).detach(), (bias - 0.1 * gb).detach()
    Wq = P.quantize_projection(W, n_heads=heads, group=64)
    lengths = [20, 7, 0]
    u = P.input_projection_q4(x[:, :L].contiguous().cuda(), Wq, bias)
    out, state, _ = P.gated_forward(u, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    got = [state.clone()]
    tokens = []
    for t in range(T):
        y, state = P.gated_layer_step(x[:, L + t].contiguous().cuda(), Wq, state, bias)
        tokens.append(y)
        got.append(state)
    V = P.dequantize_projection(Wq).cpu().double()
    for k, n in enumerate(lengths):
        seq = torch.cat([x[k, :n], x[k, L:]])
        want, _, _, _ = ref.forward(ref.project(seq, V, bias, heads).view(1, n + T, G, H))
        want = want[0]
        # pre-activations of the prompt are rounded to bf16 once: half a step of |u| <= 8 each, through slopes of at most 1/4 and
        # memories of a few steps
        for t in range(T):
            assert ((tokens[t][k].double().cpu() - want[n + t]).abs() <= 0.1).all()
            assert ((got[t + 1][k].double().cpu() - want[n + t]).abs() <= 0.1).all()
        if n == 0:
            assert (got[0][k] == 0).all()
            for t in range(T):                   # tokens alone are exact to fp32
                assert ((got[t + 1][k].double().cpu() - want[t]).abs() <= 1e-4).all()


def test_the_decode_of_a_nonlinear_cell(P):
    """4-bit pre-activations go where the projection's go: one token of the GRU."""
    gen = torch.Generator().manual_seed(95)
    Wq = P.quantize_projection(weights(3, 1, 128, seed=95).cuda(), group=32)
    x = torch.randn(4, 1, 128, generator=gen).cuda()
    params = torch.zeros(2, 3, 128, device="cuda")
    params[0].uniform_(-0.9, 0.9)
    h0 = torch.randn(4, 1, 128, device="cuda")
    u = P.input_projection_q4(x, Wq)
    h, iters, _ = P.forward("gru_diag", params, u, h0, tol=1e-5)
    a, p, s = u.double()[:, 0], params.double(), h0.double()[:, 0]
    z, r = torch.sigmoid(p[0, 0] * s + a[:, 0]), torch.sigmoid(p[0, 1] * s + a[:, 1])
    want = (1 - z) * s + z * torch.tanh(p[0, 2] * r * s + a[:, 2])
    assert iters.cpu()[1] == 0 and ((h[:, 0, 0].double() - want).abs() <= 1e-5).all()


# ---------------------------------------------------------------- refusals
def test_refusals(P):
    W = weights(2, 2, 128, seed=1).cuda()
    Wq = P.quantize_projection(W, n_heads=2, group=64)
    codes, scales = torch.zeros(2, 256, 128, dtype=torch.int8, device="cuda"), torch.ones(2, 256, 2, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(2, 3, 256, device="cuda")
    row = torch.zeros(2, 256, device="cuda")
    bad = [
        (ValueError, lambda: P.quantize_projection(W.cpu())),
        (ValueError, lambda: P.quantize_projection(W.bfloat16(), n_heads=2)),
        (ValueError, lambda: P.quantize_projection(W, n_heads=1)),
        (ValueError, lambda: P.quantize_projection(W, n_heads=0)),
        (ValueError, lambda: P.quantize_projection(W, n_heads=2, group=48)),
        (ValueError, lambda: P.quantize_projection(W, n_heads=2, group=256)),
        (ValueError, lambda: P.quantize_projection(W.transpose(0, 1), n_heads=2)),
        (ValueError, lambda: P.quantize_projection(torch.zeros(1, 96, 96, device="cuda"))),
        (ValueError, lambda: P.quantize_projection(torch.zeros(1, 64, 64, device="cuda"), group=128)),
        (ValueError, lambda: P.quantize_projection(torch.zeros(9, 64, 64, device="cuda"))),
        (ValueError, lambda: P.pack_projection(codes, scales[:, :, :1].contiguous().float(), n_heads=2)),
        (ValueError, lambda: P.pack_projection(codes, scales.cpu(), n_heads=2)),
        (ValueError, lambda: P.pack_projection(codes.int(), scales, n_heads=2)),
        (ValueError, lambda: P.pack_projection(codes, scales[0], n_heads=2)),
        (ValueError, lambda: P.input_projection_q4(x.cpu(), Wq)),
        (ValueError, lambda: P.input_projection_q4(x[0], Wq)),
        (ValueError, lambda: P.input_projection_q4(x[:, :, :128].contiguous(), Wq)),
        (ValueError, lambda: P.input_projection_q4(x, Wq, torch.zeros(3, 256, device="cuda"))),
        (KeyError, lambda: P.input_projection_q4(x.half(), Wq)),
        (RuntimeError, lambda: P.input_projection_q4(x[:0], Wq)),
        (RuntimeError, lambda: P.input_projection_q4(torch.zeros(1, P.q4_exact_rows(2048, 8, 1) + 1, 2048, device="cuda", dtype=torch.bfloat16),
                                                     P.quantize_projection(torch.zeros(8, 2048, 2048, device="cuda")),
                                                     workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
        (ValueError, lambda: P.gated_layer_step(x, Wq)),
        (ValueError, lambda: P.gated_layer_step(row, Wq, row.bfloat16())),
        (ValueError, lambda: P.gated_layer_step(row, Wq, row[:1])),
        (ValueError, lambda: P.gated_layer_step(row, P.quantize_projection(weights(1, 2, 128, seed=1).cuda(), n_heads=2))),
        (RuntimeError, lambda: P.gated_layer_step(row[:0], Wq)),
    ]
    for k, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("case", k)
    # x at an address that its 16-byte loads do not allow
    flat = torch.zeros(2 * 256 + 1, device="cuda")
    with pytest.raises(RuntimeError):
        P.gated_layer_step(flat[1:].view(2, 256), Wq)


def test_a_workspace_is_checked(P):
    """Of host memory, or of another type: refused before anything is launched."""
    Wq = P.quantize_projection(weights(2, 1, 128, seed=1).cuda())
    W = weights(2, 1, 128, seed=1).cuda()
    x = torch.zeros(1, 3, 128, device="cuda")
    u = torch.zeros(1, 3, 2, 128, device="cuda")
    host = torch.empty(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace"):
        P.input_projection_q4(x, Wq, workspace=host)
    with pytest.raises(ValueError, match="workspace"):
        P.input_projection_q4(x, Wq, workspace=torch.empty(1 << 20, device="cuda"))
    with pytest.raises(ValueError, match="workspace"):
        P.input_projection_q4(x, Wq, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(ValueError, match="workspace"):
        P.input_projection(x, W, workspace=host)
    with pytest.raises(ValueError, match="workspace"):
        P.input_projection_backward(x, W, u, workspace=host)
    assert torch.equal(P.input_projection_q4(x, Wq, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), u)
