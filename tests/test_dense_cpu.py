"""moe_decode, moe_decode_quant and the dense products: sizes and refusals, all before any HIP call (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2512_14080_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")

BIG = 1 << 40
X, WR, W1, W2, R, O, WS = (0x100000000 * i for i in range(1, 8))


def decode(D, x=X, wr=WR, bias=None, w1=W1, w2=W2, eb=None, r=R, o=O, idx=None, w=None, ws=WS, nbytes=BIG):
    return B.lib().moe_decode(D, x, wr, bias, w1, w2, eb, r, o, idx, w, ws, nbytes, None)


def test_decode_workspace():
    D = B.dims(64, 4096, 512, 128, 8)
    for which in (B.MOE_WS_DECODE, B.MOE_WS_DECODE_QUANT):
        need = B.moe_workspace_bytes(D, 0, which)
        assert need >= 64 * 8 * 4096 * 4
        assert need == B.moe_workspace_bytes(D, 12345, which)  # whatever the capacity
    for bad in ((65, 4096, 512, 128, 8), (8, 4096, 512, 1032, 8), (8, 32768, 16384, 8, 2), (0, 128, 64, 8, 2)):
        assert B.moe_workspace_bytes(B.dims(*bad), 0, B.MOE_WS_DECODE) == 0


@pytest.mark.parametrize("dims,code", [
    ((65, 128, 64, 8, 2), B.MOE_ERR_UNSUPPORTED),       # more tokens than it takes
    ((0, 128, 64, 8, 2), B.MOE_ERR_INVALID_ARG),
    ((4, 128, 64, 1032, 2), B.MOE_ERR_UNSUPPORTED),     # experts
    ((4, 32768, 16384, 8, 2), B.MOE_ERR_UNSUPPORTED),   # an expert's W1 of 2^31 bytes
    ((4, 100, 64, 8, 2), B.MOE_ERR_UNSUPPORTED),
    ((4, 128, 64, 8, 9), B.MOE_ERR_UNSUPPORTED),
])
def test_decode_refuses_sizes(dims, code):
    assert decode(B.dims(*dims)) == code, B.moe_last_error()


def test_decode_refuses_arguments():
    D = B.dims(4, 128, 64, 8, 2)
    need = B.moe_workspace_bytes(D, 0, B.MOE_WS_DECODE)
    inv = B.MOE_ERR_INVALID_ARG
    for k in ("x", "wr", "w1", "w2", "o", "ws"):
        assert decode(D, **{k: None}) == inv, k
        assert "null" in B.moe_last_error()
        assert decode(D, **{k: X + 8}) == inv, k
        assert "aligned" in B.moe_last_error()
    for k in ("bias", "idx", "w"):
        assert decode(D, **{k: X + 2}) == inv, k
    assert decode(D, r=R + 8) == inv
    assert decode(D, ws=WS + 16) == inv
    assert decode(D, nbytes=need - 1) == B.MOE_ERR_WORKSPACE
    # O over X, wholly or by a byte; over part of R
    for o in (X, X + 16, X - 16):
        assert decode(D, o=o) == inv
        assert "overlap" in B.moe_last_error()
    assert decode(D, r=O + 16) == inv
    eb = B.MoeExpertBias(X + 4, None, None, None)
    assert decode(D, eb=ctypes.byref(eb)) == inv


def test_decode_quant_refuses_weights():
    D = B.dims(4, 128, 64, 8, 2)
    L = B.lib()

    def call(q):
        return L.moe_decode_quant(D, X, WR, None, None if q is None else ctypes.byref(q), None, None, O, None, None, WS, BIG,
                                  None)

    inv = B.MOE_ERR_INVALID_ARG
    assert call(None) == inv
    q = B.MoeQExperts(128, 64, 8, B.MOE_HELD_EMPTY, W1, W1, W2, W2)
    assert call(q) == inv and "not written" in B.moe_last_error()
    q.state, q.n = B.MOE_HELD_WRITTEN, 128
    assert call(q) == inv
    q.n, q.W2s = 64, None
    assert call(q) == inv
    assert L.moe_decode_quant(B.dims(65, 128, 64, 8, 2), X, WR, None, None, None, None, O, None, None, WS, BIG,
                              None) == B.MOE_ERR_UNSUPPORTED


# ------------------------------------------------------------------ dense products
def test_linear_workspace():
    for act in B.ACTIVATIONS:
        L = B.linear_dims(1003, 904, 1528, act)
        N = 2 * 1528 if act == "swiglu" else 1528
        assert B.moe_linear_workspace_bytes(L, B.MOE_WS_LINEAR_FWD) >= 256
        assert B.moe_linear_workspace_bytes(L, B.MOE_WS_LINEAR_BWD) >= (act != "none") * 1003 * N * 2
        assert B.moe_linear_workspace_bytes(L, 3) == 0


BAD_LINEAR = [
    ((0, 64, 64, "none"), {}, B.MOE_ERR_INVALID_ARG),
    ((4, 60, 64, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    ((4, 64, 4, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    ((4, 0, 64, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    ((4, 64, 64, 5), {}, B.MOE_ERR_INVALID_ARG),
    ((4, 64, 64, -1), {}, B.MOE_ERR_INVALID_ARG),
    ((4, 1 << 24, 64, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    (((1 << 28) + 1, 8, 8, "none"), {}, B.MOE_ERR_UNSUPPORTED),  # beyond the grids' 32-bit counts
    ((1 << 28, 520, 8, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    ((1 << 28, 8, 264, "swiglu"), {}, B.MOE_ERR_UNSUPPORTED),
    ((4, (1 << 24) - 8, 1 << 15, "none"), {}, B.MOE_ERR_UNSUPPORTED),
    ((4, 64, 64, "none"), {"ldx": 56}, B.MOE_ERR_INVALID_ARG),
    ((4, 64, 64, "none"), {"ldx": 68}, B.MOE_ERR_INVALID_ARG),
    ((4, 64, 64, "none"), {"ldy": 1 << 30}, B.MOE_ERR_INVALID_ARG),
    ((4, 64, 64, "none"), {"ldr": -64}, B.MOE_ERR_INVALID_ARG),
]


@pytest.mark.parametrize("sizes,ld,code", BAD_LINEAR)
def test_linear_refuses_sizes(sizes, ld, code):
    L = B.linear_dims(*sizes, **ld)
    assert B.moe_linear_workspace_bytes(L, B.MOE_WS_LINEAR_FWD) == 0
    assert B.lib().moe_linear_fwd(L, X, W1, None, None, None, O, WS, BIG, None) == code, B.moe_last_error()
    assert B.lib().moe_linear_bwd(L, R, X, W1, W2, None, O, None, None, WS, BIG, None) == code


def test_linear_refuses_arguments():
    lib, inv = B.lib(), B.MOE_ERR_INVALID_ARG
    L = B.linear_dims(4, 64, 64, "silu")
    need = B.moe_linear_workspace_bytes(L, B.MOE_WS_LINEAR_FWD)

    def fwd(x=X, w=W1, b=None, r=None, h=None, y=O, ws=WS, nbytes=BIG):
        return lib.moe_linear_fwd(L, x, w, b, r, h, y, ws, nbytes, None)

    for k in ("x", "w", "y", "ws"):
        assert fwd(**{k: None}) == inv
        assert fwd(**{k: X + 8}) == inv
    for k in ("b", "r", "h"):
        assert fwd(**{k: X + 8}) == inv
    assert fwd(nbytes=need - 1) == B.MOE_ERR_WORKSPACE
    for y in (X, X + 16, W1 + 64):
        assert fwd(y=y) == inv and "overlap" in B.moe_last_error()
    assert fwd(h=X) == inv and fwd(h=O) == inv and fwd(r=O + 16) == inv
    need = B.moe_linear_workspace_bytes(L, B.MOE_WS_LINEAR_BWD)

    def bwd(dy=R, x=X, w=W1, h=W2, g=None, dx=O, dw=None, db=None, ws=WS, nbytes=BIG):
        return lib.moe_linear_bwd(L, dy, x, w, h, g, dx, dw, db, ws, nbytes, None)

    for k in ("dy", "w", "h", "ws"):
        assert bwd(**{k: None}) == inv, k
    assert bwd(x=None, dw=O, dx=None) == inv  # dW needs X
    assert bwd(dx=None) == inv and "all be null" in B.moe_last_error()
    for k in ("dy", "x", "w", "h", "g", "dx", "dw", "db"):
        assert bwd(**{"dw": O + (1 << 20), k: X + 8}) == inv, k
    assert bwd(nbytes=need - 1) == B.MOE_ERR_WORKSPACE
    for k, v in (("dx", R), ("dx", X), ("dx", W1), ("dw", W2), ("db", X), ("g", O + 16)):
        assert bwd(**{k: v}) == inv, (k, B.moe_last_error())
        assert "overlap" in B.moe_last_error()
    assert bwd(dw=O) == inv  # dX and dW in one place


def test_shared_expert_refuses():
    import torch
    from paper_2512_14080_amd.layer import SharedExpert
    Wu, Wd = torch.zeros(64, 48, dtype=torch.bfloat16), torch.zeros(24, 64, dtype=torch.bfloat16)
    for wu, wd in ((Wu, Wd[:, :32]), (Wu[:, :40], Wd), (Wu.t().contiguous().t(), Wd), (Wu, Wd.t().contiguous().t())):
        with pytest.raises(ValueError):
            SharedExpert(4, wu, wd)
