"""Columns and waves of the streaming 8-bit down-projection, without a GPU and each form on one, and which few tokens go by
row and token."""
import re

import pytest

from oracle import block8
from paper_2512_14080_amd import workloads as W
from test_block8_cpu import built
from test_block8_launches import _names, launches
from test_gpu_block8 import _check_o, _layer, _torch


@built
@pytest.mark.parametrize("dims,shape", [  # 16 columns each, groups of 16 rows, waves
    ((16, 1536, 256, 128, 8), (2, 1, 2)), ((10, 896, 320, 8, 8), (2, 1, 4)), ((15, 1024, 512, 8, 8), (2, 1, 4)),
    ((16, 2048, 512, 8, 8), (4, 1, 4)), ((4, 4096, 14336, 8, 2), (4, 1, 4)),
    ((64, 1024, 256, 64, 8), (8, 2, 2)), ((128, 1536, 256, 128, 8), (8, 2, 1)), ((20, 1024, 512, 16, 4), (8, 2, 4)),
    ((64, 2048, 1024, 32, 4), (8, 2, 2)), ((256, 4096, 512, 128, 8), (8, 2, 2)), ((100, 2048, 2048, 16, 1), (8, 2, 4)),
    ((64, 4096, 4096, 16, 2), (8, 2, 4)), ((20, 4096, 14336, 8, 2), (8, 2, 4)),
    ((12, 2048, 576, 16, 8), (4, 1, 4)), ((40, 640, 320, 16, 2), (8, 2, 4)), ((30, 256, 2112, 8, 2), (8, 2, 4)),
    ((20, 4224, 640, 16, 3), (8, 2, 2)),
])
def test_shape_of_the_streaming_down_projection(tmp_path, dims, shape):
    l, = launches([(dims, "quant", 0, False)], tmp_path)
    assert re.search(r"stream8_gemm_kernel.*Stream8DownELi(\d)ELi(\d)ELi(\d+)E", _names(l)).groups() == tuple(map(str, shape))


@built
@pytest.mark.parametrize("dims,by_token", [  # workgroups of the down-projection by token: T d / 32
    ((8, 4096, 64, 128, 8), True), ((16, 2048, 128, 64, 2), True), ((32, 1024, 64, 256, 8), True),
    ((16, 4096, 64, 64, 4), False), ((64, 1536, 64, 128, 2), False), ((64, 4096, 64, 128, 1), False),
    ((64, 1024, 128, 128, 2), False), ((64, 4096, 512, 128, 1), False),
])
def test_few_tokens_of_many_workgroups_go_by_expert(tmp_path, dims, by_token):
    l, = launches([(dims, "quant", 0, False)], tmp_path)
    assert ("stream8_token_down" in _names(l)) == by_token


@pytest.mark.gpu
@pytest.mark.parametrize("cfg", [
    W.MoEConfig("r12", T=12, d=2048, n=576, E=16, K=8, m_tile=16),      # (4, 1, 4): a half block at the end
    W.MoEConfig("r40", T=40, d=640, n=320, E=16, K=2, m_tile=16),       # (8, 2, 4): three blocks on four waves
    W.MoEConfig("k17", T=30, d=256, n=2112, E=8, K=2, m_tile=16, zipf_s=1.0),  # (8, 2, 4) over seventeen
    W.MoEConfig("w640", T=20, d=4224, n=640, E=16, K=3, m_tile=16),     # (8, 2, 2) over five
], ids=lambda c: c.name)
@pytest.mark.parametrize("biased", [False, True])
def test_streaming_down_projection(cfg, biased):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    inp, R, layer, b1, b2 = _layer(cfg, "quant", seed=41, biased=biased)
    layer.route()
    B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
    out = []
    for _ in range(2):
        layer.ws_f.fill_(0xFF)
        layer.O.fill_(7.0)
        B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, None, layer.O, layer.ws_f, eb=layer.eb)
        out.append(layer.O.clone())
    torch.cuda.synchronize()
    assert torch.equal(*out)
    fw = block8.forward_quant(inp.f32("X"), inp.f32("W1"), inp.f32("W2"), R, b1, b2)
    _check_o(out[0].double().cpu().numpy(), fw, R, fw["W2q"], True)
