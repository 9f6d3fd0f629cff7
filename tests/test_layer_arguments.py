"""What layer.SharedExpert and DeviceLayer.decode refuse of their tensors, before any call of the library (no GPU needed)."""
import os

import pytest
import torch

from paper_2512_14080_amd import binding as B
from paper_2512_14080_amd import workloads as W
from paper_2512_14080_amd.layer import DeviceLayer, SharedExpert

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")
T, D, M = 6, 64, 24


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _shared(T=T, **kw):
    return SharedExpert(T, _bf16(D, 2 * M), _bf16(M, D), **kw)


BAD_ROWS = {
    "fewer rows": lambda: _bf16(T - 1, D),
    "more rows": lambda: _bf16(T + 1, D),
    "other columns": lambda: _bf16(T, D + 8),
    "fp32": lambda: torch.zeros(T, D),
    "fp16": lambda: torch.zeros(T, D, dtype=torch.float16),
    "columns for rows": lambda: _bf16(D, T),
    "transposed": lambda: _bf16(D, T).t(),
    "rows apart in three dimensions": lambda: _bf16(2, T // 2, D + 8)[..., :D],
    "every other column": lambda: _bf16(T, 2 * D)[:, ::2],
    "one row for all": lambda: _bf16(1, D).expand(T, D),
    "rows that overlap": lambda: _bf16(T * D).as_strided((T, D), (D - 8, 1)),
    "another device": lambda: torch.empty((T, D), dtype=torch.bfloat16, device="meta"),
}


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_shared_expert_refuses_rows(bad):
    s, good, t = _shared(train=True), _bf16(T, D), BAD_ROWS[bad]()
    for args in ((t, good), (good, t), (good, good, t)):
        with pytest.raises(ValueError, match="^(X|Y|R) must be|^the rows of (X|Y|R) must"):
            s.forward(*args)
    for args in ((t, good, good), (good, t, good), (good, good, t), (good, good, good, t)):
        with pytest.raises(ValueError, match="^(dY|X|dX|G) must be|^the rows of (dY|X|dX|G) must"):
            s.backward(*args)


def test_shared_expert_refuses_unlike_strides_of_x():
    """X, dX and G have one stride in the library's call."""
    s, good, wide = _shared(train=True), _bf16(T, D), _bf16(T, D + 8)[:, :D]
    for args in ((good, good, wide), (good, wide, good), (good, good, good, wide)):
        with pytest.raises(ValueError, match="equally far apart"):
            s.backward(*args)


def test_shared_expert_needs_a_gpu():
    s, good, wide = _shared(train=True), _bf16(T, D), _bf16(T, D + 8)[:, :D]
    for x in (good, wide, good.view(2, -1, D), good.view(-1)):
        with pytest.raises(ValueError, match="must be on a GPU"):
            s.forward(x, good, wide)
        with pytest.raises(ValueError, match="must be on a GPU"):
            s.backward(wide, x, x, x)
    one = _shared(1)  # (one row: its stride means nothing)
    with pytest.raises(ValueError, match="must be on a GPU"):
        one.forward(_bf16(D, 1).t(), _bf16(1, D))


def test_shared_expert_workspace_holds_any_stride():
    for t, d, m in ((1, 64, 24), (16, 8192, 256), (64, 4096, 512), (300, 16384, 64)):
        s = SharedExpert(t, _bf16(d, 2 * m), _bf16(m, d), train=True)
        for ld in (0, d + 8, (1 << 30) - 8):
            assert s.ws_f.numel() >= B.moe_linear_workspace_bytes(B.linear_dims(t, d, m, "swiglu", ldx=ld), B.MOE_WS_LINEAR_FWD)
            assert s.ws_b.numel() >= B.moe_linear_workspace_bytes(B.linear_dims(t, d, m, "swiglu", ldx=ld), B.MOE_WS_LINEAR_BWD)
            down = B.linear_dims(t, m, d, ldr=ld, ldy=ld)
            assert s.ws_f.numel() >= B.moe_linear_workspace_bytes(down, B.MOE_WS_LINEAR_FWD)
            assert s.ws_b.numel() >= B.moe_linear_workspace_bytes(down, B.MOE_WS_LINEAR_BWD)


@pytest.mark.parametrize("name,bad", [
    ("bu", lambda: _bf16(2 * M)), ("bu", lambda: torch.zeros(M)), ("bu", lambda: torch.zeros(2 * M, dtype=torch.float64)),
    ("bu", lambda: torch.zeros(4 * M)[::2]), ("bu", lambda: torch.zeros(1).expand(2 * M)), ("bu", lambda: torch.zeros(M, 2)),
    ("bd", lambda: _bf16(D)), ("bd", lambda: torch.zeros(D - 8)), ("bd", lambda: torch.zeros(D, device="meta")),
    ("Wu", lambda: torch.zeros(D, 2 * M)), ("Wd", lambda: torch.zeros(M, D, dtype=torch.float16)),
    ("Wd", lambda: torch.empty((M, D), dtype=torch.bfloat16, device="meta")),
])
def test_shared_expert_refuses_weights_and_biases(name, bad):
    args = {"Wu": _bf16(D, 2 * M), "Wd": _bf16(M, D), "bu": torch.zeros(2 * M), "bd": torch.zeros(D)}
    SharedExpert(T, **args)
    with pytest.raises(ValueError, match=name):
        SharedExpert(T, **{**args, name: bad()})


def test_shared_expert_backward_needs_train():
    with pytest.raises(ValueError, match="train=True"):
        _shared().backward(_bf16(T, D), _bf16(T, D), _bf16(T, D))


# ------------------------------------------------------------------ decode
CFG = W.MoEConfig("decode", T=5, d=128, n=64, E=8, K=2, m_tile=64)


def _layer(**kw):
    return DeviceLayer(W.make_inputs(CFG, 3), device="cpu", **kw)


BAD_DECODE = {
    "R of fewer rows": lambda: {"R": _bf16(4, 128)},
    "R of other columns": lambda: {"R": _bf16(5, 64)},
    "R in fp32": lambda: {"R": torch.zeros(5, 128)},
    "R with rows apart": lambda: {"R": _bf16(5, 136)[:, :128]},
    "one row of R for all": lambda: {"R": _bf16(1, 128).expand(5, 128)},
    "R elsewhere": lambda: {"R": torch.empty((5, 128), dtype=torch.bfloat16, device="meta")},
    "topk_idx in 64 bits": lambda: {"topk_idx": torch.zeros((5, 2), dtype=torch.int64)},
    "topk_idx of fewer rows": lambda: {"topk_idx": torch.zeros((4, 2), dtype=torch.int32)},
    "topk_idx of one column": lambda: {"topk_idx": torch.zeros((5, 1), dtype=torch.int32)},
    "topk_w in bf16": lambda: {"topk_w": _bf16(5, 2)},
    "topk_w transposed": lambda: {"topk_w": torch.zeros((2, 5)).t()},
}


@pytest.mark.parametrize("bad", BAD_DECODE)
def test_decode_refuses_tensors(bad):
    kw = BAD_DECODE[bad]()
    with pytest.raises(ValueError, match=f"{next(iter(kw))} must be"):
        _layer().decode(**kw)


def test_decode_needs_a_gpu():
    with pytest.raises(ValueError, match="must be on a GPU"):
        _layer().decode(_bf16(5, 128), topk_idx=torch.zeros((5, 2), dtype=torch.int32), topk_w=torch.zeros((5, 2)))


def test_decode_refuses_given_scores():
    """route and step go by the scores given to the layer, which the call cannot take."""
    import numpy as np
    scores = np.random.default_rng(0).random((5, 8), np.float32)
    with pytest.raises(ValueError, match="scores_in"):
        _layer(scores_in=scores).decode()


def test_decode_takes_no_memory_in_a_call():
    """A workspace made in a call on another stream than the current one would be memory that the current one may still be
    writing for someone else."""
    D = B.dims(5, 128, 64, 8, 2)
    assert _layer().ws_d.numel() == B.moe_workspace_bytes(D, 10, B.MOE_WS_DECODE)
    assert _layer(held8="quant").ws_d.numel() == B.moe_workspace_bytes(D, 10, B.MOE_WS_DECODE_QUANT)
    assert _layer(round_mode="nearest").ws_d is None
    long = W.MoEConfig("decode", T=65, d=128, n=64, E=8, K=2, m_tile=64)
    assert DeviceLayer(W.make_inputs(long, 3), device="cpu").ws_d.numel() == 0  # (the call refuses T)
