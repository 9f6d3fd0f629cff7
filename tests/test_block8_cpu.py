"""The 8-bit operators without a GPU: the oracle's format against torch's e4m3 type and the definition, the entry
points' sizes and refusals, and the kernels that their rules choose."""
import ctypes
import os

import numpy as np
import pytest
import torch

import oracle
from oracle import block8
from paper_2512_14080_amd import binding as B
from test_abi_cpu import _fake_routing

built = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")
PTR = 0x100000  # non-null and aligned; validation only inspects it


def test_codes_are_those_of_the_e4m3_type():
    """Every code's value, and rounding at, next to and between all of them, as torch's float8_e4m3fn has it."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(block8.VALUES, every)
    pos = block8.VALUES[:0x7F]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64),
                        np.nextafter(mid.astype(np.float32), np.float32(500)).astype(np.float64)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(block8.encode(x), want)


def test_a_scale_is_the_least_that_holds_its_block():
    x = np.zeros((8, 256))
    x[0, :3] = [448.0, -1.0, 3.0]
    x[1, 130] = np.nextafter(448.0, 500)
    x[2, 5] = 2.0 ** -140
    x[3, 0], x[3, 200] = np.inf, np.nan
    x[4, 0], x[4, 1] = 3.38e38, np.inf
    q, e, v = block8.quantize(x)
    assert e[0, 0] == 0 and e[0, 1] == -126 and e[1, 1] == 1 and e[2, 0] == -126
    assert (e[3] == -126).all() and q[3, 0] == 0x7F and q[3, 200] == 0x7F and np.isnan(v[3, 0])
    assert e[4, 0] == 120 and v[4, 0] == 3.38e38 or abs(v[4, 0] / 3.38e38 - 1) <= 2 ** -4


def test_a_value_is_off_by_at_most_half_a_step():
    x = np.random.default_rng(0).standard_normal((64, 333)) * np.exp(np.random.default_rng(1).uniform(-30, 30, (64, 1)))
    q, e, v = block8.quantize(x)
    s = np.ldexp(1.0, np.repeat(e, 128, 1)[:, :333])
    assert (np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)).all()


# ------------------------------------------------------------------ sizes and refusals
@built
def test_scale_stride():
    assert [B.scale_stride(c) for c in (-8, 0, 1, 128, 512, 513, 1024, 1032)] == [0, 0, 4, 4, 4, 8, 8, 12]
    assert B.scale_stride(2 ** 31 - 1) == 2 ** 24


@built
@pytest.mark.parametrize("rows,cols,code", [(-1, 128, B.MOE_ERR_INVALID_ARG), (4, 0, B.MOE_ERR_UNSUPPORTED),
                                            (4, 12, B.MOE_ERR_UNSUPPORTED), (4, -8, B.MOE_ERR_UNSUPPORTED),
                                            (1 << 31, 8, B.MOE_ERR_UNSUPPORTED), (1 << 30, 264, B.MOE_ERR_UNSUPPORTED),
                                            (1 << 62, 1024, B.MOE_ERR_UNSUPPORTED), (0, 128, B.MOE_OK)])
def test_rows_sizes_refused(rows, cols, code):
    L = B.lib()
    assert L.moe_quantize_rows(rows, cols, PTR, PTR, PTR, None) == code, B.moe_last_error()
    assert L.moe_dequantize_rows(rows, cols, PTR, PTR, PTR, None) == code


@built
def test_rows_pointers_refused():
    L = B.lib()
    for X, q, s in ((None, PTR, PTR), (PTR, None, PTR), (PTR, PTR, None), (PTR + 8, PTR, PTR), (PTR, PTR + 4, PTR),
                    (PTR, PTR, PTR + 2)):
        assert L.moe_quantize_rows(4, 128, X, q, s, None) == B.MOE_ERR_INVALID_ARG
        assert L.moe_dequantize_rows(4, 128, q, s, X, None) == B.MOE_ERR_INVALID_ARG


def _qexperts(D, state=B.MOE_HELD_WRITTEN):
    q = B.MoeQExperts()
    nbytes = B.lib().moe_qexperts_bytes(D)
    assert B.lib().moe_qexperts_init(D, PTR, nbytes, ctypes.byref(q)) == B.MOE_OK
    assert q.state == B.MOE_HELD_EMPTY
    q.state = state
    return q


def _ckpt(D, capacity, flags=0, state=B.MOE_HELD_WRITTEN):
    c = B.MoeCkpt()
    nbytes = B.lib().moe_ckpt_bytes(D, capacity, flags)
    assert B.lib().moe_ckpt_init(D, capacity, flags, PTR, nbytes, ctypes.byref(c)) == B.MOE_OK
    assert c.state == B.MOE_HELD_EMPTY and bool(c.X) == bool(c.Xs) == bool(flags)
    c.state = state
    return c


@built
def test_buffers():
    D = B.dims(1000, 384, 192, 16, 4)
    L = B.lib()
    # n = 192 is padded to 256 columns
    assert L.moe_qexperts_bytes(D) >= 16 * 3 * 384 * 256
    assert L.moe_ckpt_bytes(D, 4000, 0) >= 4000 * (2 * 192 + 4)
    assert L.moe_ckpt_bytes(D, 4000, B.MOE_CKPT_X) >= L.moe_ckpt_bytes(D, 4000, 0) + 1000 * (384 + 4)
    assert L.moe_ckpt_bytes(D, 0, 0) == 0 and L.moe_ckpt_bytes(D, 4000, 2) == 0
    assert L.moe_ckpt_bytes(B.dims(0, 384, 192, 16, 4), 4000, 0) == 0
    assert L.moe_qexperts_bytes(B.dims(1, 100, 192, 16, 4)) == 0
    q, c = B.MoeQExperts(), B.MoeCkpt()
    need = L.moe_qexperts_bytes(D)
    assert L.moe_qexperts_init(D, PTR, need - 1, ctypes.byref(q)) == B.MOE_ERR_INVALID_ARG
    assert L.moe_qexperts_init(D, PTR + 128, need, ctypes.byref(q)) == B.MOE_ERR_INVALID_ARG
    assert L.moe_qexperts_init(D, None, need, ctypes.byref(q)) == B.MOE_ERR_INVALID_ARG
    need = L.moe_ckpt_bytes(D, 4000, 0)
    assert L.moe_ckpt_init(D, 4000, 0, PTR, need - 1, ctypes.byref(c)) == B.MOE_ERR_INVALID_ARG
    assert L.moe_ckpt_init(D, 0, 0, PTR, need, ctypes.byref(c)) == B.MOE_ERR_CAPACITY
    assert L.moe_ckpt_init(D, 4000, 6, PTR, need, ctypes.byref(c)) == B.MOE_ERR_INVALID_ARG
    for which in (B.MOE_WS_FWD_QUANT, B.MOE_WS_FWD_CKPT, B.MOE_WS_BWD_CKPT):
        assert B.moe_workspace_bytes(D, 4000, which) > 0
    assert B.moe_workspace_bytes(D, 4000, B.MOE_WS_BWD_CKPT) >= B.moe_workspace_bytes(D, 4000, B.MOE_WS_BWD) + 1000 * 768


D0 = (256, 128, 64, 8, 2)


def _quant_args(D, **kw):
    r = kw.get("r", _fake_routing(D, 512))
    q = kw.get("q", _qexperts(D))
    c = kw.get("c")
    ws = kw.get("ws", B.moe_workspace_bytes(D, 512, B.MOE_WS_FWD_QUANT))
    ref = lambda x: None if x is None else ctypes.byref(x)
    return [D, kw.get("X", PTR), ref(q), None, ref(r), ref(c), kw.get("O", PTR), kw.get("wsp", PTR), ws, None]


@built
def test_quantized_forward_refusals():
    D, L = B.dims(*D0), B.lib()

    def refused(code, word, **kw):
        assert L.moe_fwd_quant(*_quant_args(D, **kw)) == code, kw
        assert word in B.moe_last_error(), B.moe_last_error()

    refused(B.MOE_ERR_INVALID_ARG, "8-bit weights", q=None)
    refused(B.MOE_ERR_INVALID_ARG, "not written", q=_qexperts(D, B.MOE_HELD_EMPTY))
    refused(B.MOE_ERR_INVALID_ARG, "n = 128", q=_qexperts(B.dims(256, 128, 128, 8, 2)))
    refused(B.MOE_ERR_INVALID_ARG, "E = 16", q=_qexperts(B.dims(256, 128, 64, 16, 2)))
    refused(B.MOE_ERR_INVALID_ARG, "capacity 600", c=_ckpt(D, 600))
    refused(B.MOE_ERR_INVALID_ARG, "X", X=None)
    refused(B.MOE_ERR_INVALID_ARG, "O", O=PTR + 8)
    refused(B.MOE_ERR_WORKSPACE, "workspace", ws=B.moe_workspace_bytes(D, 512, B.MOE_WS_FWD_QUANT) - 1)
    refused(B.MOE_ERR_INVALID_ARG, "ws", wsp=None)
    r = _fake_routing(D, 512)
    r.state = B.MOE_ROUTING_STATE_COUNTS
    refused(B.MOE_ERR_INVALID_ARG, "not a complete routing", r=r)


@built
def test_checkpointed_calls_refusals():
    D, L = B.dims(*D0), B.lib()
    r = _fake_routing(D, 512)
    wf, wb = (B.moe_workspace_bytes(D, 512, w) for w in (B.MOE_WS_FWD_CKPT, B.MOE_WS_BWD_CKPT))

    def fwd(c, ws=wf, X=PTR):
        return L.moe_fwd_ckpt(D, X, PTR, PTR, None, ctypes.byref(r), None if c is None else ctypes.byref(c), PTR, PTR, ws, None)

    def bwd(c, ws=wb, X=PTR, Wr=PTR):
        return L.moe_bwd_ckpt(D, PTR, X, None if c is None else ctypes.byref(c), PTR, PTR, None, Wr, ctypes.byref(r), PTR,
                              PTR, PTR, PTR, PTR, None, PTR, ws, None)

    assert fwd(None) == bwd(None) == B.MOE_ERR_INVALID_ARG
    other = _ckpt(B.dims(255, 128, 64, 8, 2), 512)
    assert fwd(other) == bwd(other) == B.MOE_ERR_INVALID_ARG and "T = 255" in B.moe_last_error()
    assert fwd(_ckpt(D, 512), X=None) == B.MOE_ERR_INVALID_ARG
    assert fwd(_ckpt(D, 512), ws=wf - 1) == B.MOE_ERR_WORKSPACE
    assert bwd(_ckpt(D, 512, state=B.MOE_HELD_EMPTY)) == B.MOE_ERR_INVALID_ARG and "not written" in B.moe_last_error()
    assert bwd(_ckpt(D, 512), X=None) == B.MOE_ERR_INVALID_ARG and "MOE_CKPT_X" in B.moe_last_error()
    assert bwd(_ckpt(D, 512), X=PTR + 2) == B.MOE_ERR_INVALID_ARG
    assert bwd(_ckpt(D, 512), ws=wb - 1) == B.MOE_ERR_WORKSPACE
    assert bwd(_ckpt(D, 512), Wr=None) == B.MOE_ERR_INVALID_ARG and "Wr" in B.moe_last_error()
    c = _ckpt(D, 512)
    c.Hs = None
    assert bwd(c) == B.MOE_ERR_INVALID_ARG and "null array" in B.moe_last_error()


@built
def test_experts_refusals():
    D, L = B.dims(*D0), B.lib()
    q, empty = _qexperts(D), _qexperts(D, B.MOE_HELD_EMPTY)
    assert L.moe_quantize_experts(D, PTR, None, ctypes.byref(q), None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_quantize_experts(D, PTR + 8, PTR, ctypes.byref(q), None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_quantize_experts(D, PTR, PTR, None, None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_dequantize_experts(D, ctypes.byref(empty), PTR, PTR, None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_dequantize_experts(B.dims(256, 256, 64, 8, 2), ctypes.byref(q), PTR, PTR, None) == B.MOE_ERR_INVALID_ARG


def test_gradient_formula_against_differences():
    """The oracle's backward from kept H and X, in 64 bits, against central differences of the forward whose H is that
    value: exact where H is kept exactly (no rounding on the way)."""
    rng = np.random.default_rng(3)
    T, d, n, E, K = 6, 8, 4, 3, 2
    X, W1, W2, Wr, dO = (rng.standard_normal(s) for s in ((T, d), (E, d, 2 * n), (E, n, d), (d, E), (T, d)))
    idx = np.argsort(-(X @ Wr), 1)[:, :K]
    member = np.zeros((T, E), bool)
    np.put_along_axis(member, idx, True, 1)

    def loss(X, W1, W2, Wr):
        S = oracle.softmax_scores(X @ Wr)
        R = oracle.routing_from_membership(member, S, np.float64)
        return (oracle.forward(X, W1, W2, R, dtype=np.float64)["O"] * dO).sum(), R

    _, R = loss(X, W1, W2, Wr)
    H = oracle.forward(X, W1, W2, R, dtype=np.float64)["H"]
    g = block8.backward_ckpt(dO, X, H, W1, W2, Wr, R)
    for name, i, at in (("dX", 0, (2, 3)), ("dW1", 1, (1, 2, 5)), ("dW2", 2, (0, 1, 4)), ("dWr", 3, (3, 1))):
        args = [[a.copy() for a in (X, W1, W2, Wr)] for _ in range(2)]
        args[0][i][at] += 1e-6
        args[1][i][at] -= 1e-6
        diff = (loss(*args[0])[0] - loss(*args[1])[0]) / 2e-6
        assert abs(diff - g[name][at]) <= 1e-6 * max(1, abs(diff)), name


@pytest.mark.parametrize("kw", [{"held8": "fp8"}, {"held8": True}, {"keep_x": True}])
def test_layer_refuses(kw):
    from paper_2512_14080_amd.layer import DeviceLayer
    with pytest.raises(ValueError):
        DeviceLayer(None, **kw)
