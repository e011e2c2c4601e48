"""Host-side checks of the gated linear recurrence and of 4-bit weights that need no GPU: sizes, and the refusals that come
before any device work (through the C ABI, with addresses that are never read)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_21450_amd", "libpararnn.so")
F32, BF16 = 0, 1
INVALID, TOO_SMALL, UNSUPPORTED = 2, 3, 6
A = 1 << 20                      # an aligned address


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2510_21450_amd import build
        build.build()
    lib = ctypes.CDLL(LIB)
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    for name, res, args in (("gated_workspace_bytes", sz, [i] * 5), ("gated_checkpoint_bytes", sz, [i] * 5),
                            ("gated_forward", i, [i, vp, vp, vp, i, i, i, i, vp, vp, vp, vp, sz, vp]),
                            ("gated_backward", i, [i, vp, vp, vp, vp, vp, i, i, i, i, vp, vp, vp, sz, vp]),
                            ("q4_packed_bytes", sz, [i] * 3), ("q4_scale_bytes", sz, [i] * 4), ("q4_workspace_bytes", sz, [i] * 7),
                            ("q4_exact_rows", i, [i] * 3), ("q4_quantize", i, [vp, i, i, i, i, vp, vp, vp]),
                            ("q4_pack", i, [vp, vp, i, i, i, i, vp, vp, vp]), ("q4_dequantize", i, [vp, vp, i, i, i, i, vp, vp]),
                            ("input_projection_q4", i, [i, vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, sz, vp]),
                            ("gated_layer_step", i, [i, vp, vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp])):
        f = getattr(lib, "pararnn_" + name)
        f.restype, f.argtypes = res, args
    return lib


def test_gated_sizes(lib):
    ws, ck = lib.pararnn_gated_workspace_bytes, lib.pararnn_gated_checkpoint_bytes
    for f in (ws, ck):
        assert f(2, 1, 1, 1, 2) == 0 and f(F32, 0, 1, 1, 2) == 0 and f(F32, 1, 0, 1, 2) == 0 and f(F32, 1, 1, 0, 2) == 0
        assert f(F32, 1, 1, 1, 1) == 0 and f(F32, 1, 1, 1, 4) == 0 and f(F32, 1, 1, (1 << 20) + 1, 2) == 0
    for dtype in (F32, BF16):
        assert ws(dtype, 3, 1, 1000, 3) >= 256 and ws(dtype, 3, 1, 1000, 3) % 256 == 0
        assert ck(dtype, 3, 1, 1000, 3) == 3 * 1000 * 4
        rows = ck(dtype, 2, 10000, 8, 2) // (2 * 8 * 4)
        assert ck(dtype, 2, 10000, 8, 2) == rows * 2 * 8 * 4 and 10000 / 512 <= rows <= 10000 / 16
    # states between the checkpoints are a small part of the states
    assert ck(BF16, 4, 65536, 4096, 2) <= 4 * 65536 * 4096 * 2 // 16


def test_gated_refusals(lib):
    fwd, bwd = lib.pararnn_gated_forward, lib.pararnn_gated_backward
    n = 1 << 30

    def forward(dtype=F32, u=A, h0=A, lengths=A, B=2, L=3000, H=64, G=2, h=A, last=A, ck=A, ws=A, bytes=n):
        return fwd(dtype, u, h0, lengths, B, L, H, G, h, last, ck, ws, bytes, None)

    def backward(dtype=F32, u=A, ck=A, lengths=A, g=A, dlast=A, B=2, L=3000, H=64, G=2, du=A, dh0=A, ws=A, bytes=n):
        return bwd(dtype, u, ck, lengths, g, dlast, B, L, H, G, du, dh0, ws, bytes, None)
    for call in (forward, backward):
        for kw in (dict(dtype=2), dict(u=None), dict(B=0), dict(L=-1), dict(H=0), dict(G=1), dict(G=4), dict(ws=None), dict(ws=A + 16),
                   dict(u=A + 2), dict(lengths=A + 2)):
            assert call(**kw) == INVALID, (call, kw)
        assert call(H=(1 << 20) + 1) == UNSUPPORTED
        # more tiles, or channels of all sequences, than a launch has threads for
        assert call(B=1 << 23, L=1, H=64, bytes=1 << 60) == UNSUPPORTED and call(B=1 << 14, L=129 << 13, H=1, bytes=1 << 60) == UNSUPPORTED
        assert call(B=1 << 13, L=1, H=1 << 20, bytes=1 << 60) == UNSUPPORTED
        assert call(bytes=lib.pararnn_gated_workspace_bytes(F32, 2, 3000, 64, 2) - 1) == TOO_SMALL
        assert call(dtype=BF16, u=A + 1) == INVALID
    for kw in (dict(h=None), dict(h=A + 2), dict(h0=A + 2), dict(last=A + 2), dict(ck=A + 2)):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(du=None), dict(ck=None), dict(du=A + 2), dict(g=A + 2), dict(dlast=A + 2), dict(dh0=A + 2), dict(ck=A + 2)):
        assert backward(**kw) == INVALID, kw


def test_q4_sizes(lib):
    assert lib.pararnn_q4_packed_bytes(256, 3, 2) == 3 * 256 * 128 // 2
    assert lib.pararnn_q4_scale_bytes(256, 3, 2, 64) == 3 * 256 * 2 * 2
    for H, G, heads in ((0, 1, 1), (64, 0, 1), (64, 9, 1), (64, 1, 0), (100, 1, 1), (128, 1, 3), (96, 1, 1), (1 << 21, 1, 1 << 15)):
        assert lib.pararnn_q4_packed_bytes(H, G, heads) == 0 and lib.pararnn_q4_exact_rows(H, G, heads) == -1, (H, G, heads)
    for group in (0, 16, 48, 128):
        assert lib.pararnn_q4_scale_bytes(64, 1, 1, group) == 0
    ws = lib.pararnn_q4_workspace_bytes
    few = lib.pararnn_q4_exact_rows(4096, 3, 1)
    assert 64 <= few < 4000 and lib.pararnn_q4_exact_rows(128, 2, 1) >= 64
    assert ws(BF16, 1, few, 4096, 3, 1, 64) == 256 and ws(BF16, few + 1, 1, 4096, 3, 1, 64) >= 3 * 4096 * 4096 * 2
    assert ws(F32, 1, few + 1, 256, 2, 1, 64) >= 256
    assert ws(2, 1, 1, 256, 2, 1, 64) == 0 and ws(BF16, 0, 1, 256, 2, 1, 64) == 0 and ws(BF16, 1, 1, 256, 2, 1, 48) == 0


def test_q4_refusals(lib):
    def quantize(W=A, H=128, G=2, heads=1, group=64, packed=A, scales=A):
        return lib.pararnn_q4_quantize(W, H, G, heads, group, packed, scales, None)

    def pack(W=A, cs=A, H=128, G=2, heads=1, group=64, packed=A, scales=A):
        return lib.pararnn_q4_pack(W, cs, H, G, heads, group, packed, scales, None)

    def dequantize(W=A, H=128, G=2, heads=1, group=64, packed=A, scales=A):
        return lib.pararnn_q4_dequantize(packed, scales, H, G, heads, group, W, None)

    def project(dtype=F32, x=A, packed=A, scales=A, bias=A, B=2, L=3, H=128, G=2, heads=1, group=64, u=A, ws=A, bytes=1 << 30):
        return lib.pararnn_input_projection_q4(dtype, x, packed, scales, bias, B, L, H, G, heads, group, u, ws, bytes, None)

    def step(dtype=F32, x=A, packed=A, scales=A, bias=A, h=A, B=2, H=128, G=2, heads=1, group=64, y=A, nxt=A):
        return lib.pararnn_gated_layer_step(dtype, x, packed, scales, bias, h, B, H, G, heads, group, y, nxt, None)
    for call in (quantize, pack, dequantize, project, step):
        for kw in (dict(packed=None), dict(packed=A + 8), dict(scales=None), dict(scales=A + 1), dict(H=0), dict(G=0), dict(G=9),
                   dict(heads=0), dict(heads=3), dict(group=0), dict(group=96)):
            assert call(**kw) == INVALID, (call, kw)
        for kw in (dict(H=96), dict(H=192, group=128), dict(H=1 << 21, heads=1 << 14, group=32), dict(H=1 << 18, G=3)):
            assert call(**kw) == UNSUPPORTED, (call, kw)
    for call in (quantize, pack, dequantize):
        assert call(W=None) == INVALID
    assert quantize(W=A + 2) == INVALID and dequantize(W=A + 2) == INVALID and pack(cs=A + 1) == INVALID and pack(cs=None) == INVALID
    for call in (project, step):
        for kw in (dict(dtype=2), dict(x=None), dict(x=A + 8), dict(bias=A + 2), dict(B=0)):
            assert call(**kw) == INVALID, (call, kw)
    assert project(L=0) == INVALID and project(u=A + 2) == INVALID and project(u=None) == INVALID and project(ws=A + 8) == INVALID
    many = dict(dtype=BF16, B=1, L=lib.pararnn_q4_exact_rows(4096, 3, 1) + 1, H=4096, G=3)
    assert project(bytes=256, **many) == TOO_SMALL and project(u=A + 2, **many) == UNSUPPORTED
    assert step(G=1) == INVALID and step(G=4) == INVALID and step(y=None) == INVALID and step(nxt=None) == INVALID
    assert project(B=1 << 10, L=1 << 19, H=1 << 14, heads=1 << 8) == UNSUPPORTED        # more workgroups than a launch has
    assert step(h=A + 2) == INVALID and step(nxt=A + 2) == INVALID and step(B=(1 << 20) + 1) == UNSUPPORTED


def test_choice_of_products(lib):
    """What a call asks of its workspace and of u is the same in either mode; other modes do not exist."""
    few = lib.pararnn_q4_exact_rows(4096, 3, 1)
    assert lib.pararnn_set_q4_products(-1) == INVALID and lib.pararnn_set_q4_products(2) == INVALID
    asked = []
    for mode in (0, 1, 0):
        assert lib.pararnn_set_q4_products(mode) == 0
        many = (BF16, A, A, A, A, 1, few + 1, 4096, 3, 1, 64)
        asked.append((lib.pararnn_q4_exact_rows(4096, 3, 1), lib.pararnn_q4_workspace_bytes(BF16, 1, few + 1, 4096, 3, 1, 64),
                      lib.pararnn_input_projection_q4(*many, A, A, 256, None), lib.pararnn_input_projection_q4(*many, A + 2, A, 1 << 30, None)))
    assert asked[0] == asked[1] == asked[2] and asked[0][2:] == (TOO_SMALL, UNSUPPORTED)
    try:
        assert lib.pararnn_set_q4_products(1) == 0 and lib.pararnn_q4_products() == 1
        assert lib.pararnn_input_projection_q4(BF16, A, A, A, A, 1, few + 1, 4096, 3, 1, 64, A, None, 0, None) == INVALID
    finally:
        assert lib.pararnn_set_q4_products(0) == 0 and lib.pararnn_q4_products() == 0


def test_python_refuses_what_is_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    import paper_2510_21450_amd as P
    u = torch.zeros(1, 2, 2, 8)
    for call in (lambda: P.gated_forward(u), lambda: P.gated_backward(u, u), lambda: P.gated_apply(u),
                 lambda: P.quantize_projection(torch.zeros(1, 64, 64)), lambda: P.pack_projection(torch.zeros(1, 64, 64), u),
                 lambda: P.gated_layer(torch.zeros(1, 2, 64), torch.zeros(2, 64, 64))):
        with pytest.raises(ValueError):
            call()
