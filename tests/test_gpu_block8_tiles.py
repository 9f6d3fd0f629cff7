"""The 8-bit up-projection that keeps H, where a workgroup computes several full tiles and the last block of n is a half.

A wave whose columns lie past n stores less than the others behind a tile that counts as full, and the next tile's first
wait counts stores.  H is compared with its products in 64 bits, O with that of the call that keeps nothing.
"""
import pytest

from test_block8_cpu import built
from test_block8_launches import _names, launches
from test_gpu_block8_accuracy import OFF
from test_gpu_parity import _torch

# (dims, m_tile of a rounding up or 0, rows of the up-projection's tiles)
CASES = [
    ((50000, 384, 192, 8, 2), 0, 256),
    ((50000, 512, 64, 8, 4), 0, 256),
    ((14000, 512, 192, 512, 4), 128, 128),
    ((28000, 384, 64, 1024, 4), 128, 128),
]


@built
@pytest.mark.parametrize("dims,m_tile,rows", CASES)
def test_tiles_of_the_cases(tmp_path, dims, m_tile, rows):
    l, = launches([(dims, "kept", m_tile, False)], tmp_path)
    assert f"OpUp8INS_7GemmCfgILi{rows}ELi256E" in _names(l)


def _far_off(torch, H, ref, terms):
    """Kept values H that are further from the 64-bit ref than the products' error (terms) and one step of its block."""
    block = torch.nn.functional.max_pool1d(ref.abs()[None], 128, ceil_mode=True)[0].repeat_interleave(128, 1)[:, :ref.shape[1]]
    # a step is at most 2^-3 of the value, or 2^-9 of a scale, which is at most amax / 224
    return ((H - ref).abs() > terms + torch.maximum(ref.abs() / 8, (block + terms.amax()) * (2.0 ** -9 / 224))).sum()


@pytest.mark.gpu
@pytest.mark.parametrize("dims,m_tile,rows", CASES)
def test_several_full_tiles_of_a_half_block(dims, m_tile, rows):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    T, d, n, E, K = dims
    D = B.dims(*dims)
    g = torch.Generator(device="cuda").manual_seed(n + rows)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    X, W1, W2 = normal(T, d), normal(E, d, 2 * n, std=0.05), normal(E, n, d, std=0.05)
    b1 = torch.randn((E, 2 * n), generator=g, device="cuda")
    r = B.Routing(D, T * K, B.MOE_ROUTING_SCORES_T if m_tile else 0)
    r.arrays()["scores"].copy_(torch.softmax(torch.randn((T, E), generator=g, device="cuda"), 1))
    B.moe_route(D, None, None, None, B.MOE_ROUTE_SCORES_IN | (B.MOE_ROUTE_WRITE_SCORES_T if m_tile else 0), r)
    if m_tile:
        tc, r = r, B.Routing(D, B.moe_round_capacity(D, m_tile))
        B.moe_round_tokens(D, m_tile, "up", None, tc, r)
    counts = r.arrays()["counts"].tolist()
    tiles = sum(-(-c // rows) for c in counts) * -(-n // 128)
    full = sum(c // rows for c in counts) * -(-n // 128)
    assert tiles > 3 * 256 and full > 0.9 * tiles, (tiles, full)

    qw = B.QExperts(D)
    B.moe_quantize_experts(D, W1, W2, qw)
    B.moe_dequantize_experts(D, qw, W1, W2)  # the values that the codes stand for
    ckpt = B.Checkpoint(D, r.capacity, keep_x=True)
    ws = torch.empty(B.moe_workspace_bytes(D, r.capacity, B.MOE_WS_FWD_QUANT), dtype=torch.uint8, device="cuda")
    eb = B.expert_bias(b1, None)
    out = []
    for c in (ckpt, None, ckpt):
        ws.fill_(0xFF)
        O = torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_fwd_quant(D, X, qw, r, c, O, ws, eb=eb)
        out.append((O, {k: v.clone() for k, v in ckpt.arrays().items()}))
    torch.cuda.synchronize()
    assert torch.equal(out[0][0], out[2][0])
    # without a checkpoint: other sums, and so a few other codes of A
    kept, plain = (out[i][0].double() for i in (0, 1))
    assert ((kept - plain).norm() / plain.norm()).item() <= 2 * OFF["tiled"]
    first = int(r.arrays()["offsets"][E])
    for k in ("H", "Hs"):
        assert torch.equal(out[0][1][k][:first], out[2][1][k][:first]), k

    a = out[0][1]
    nb = -(-n // 128)
    x8 = torch.empty_like(X)
    B.moe_dequantize_rows(T, d, a["X"], a["Xs"], x8)
    x8 = x8.double()
    token, at, bad = r.arrays()["row_token"].long(), 0, 0
    for e in range(E):
        rows_e = slice(at, at + counts[e])
        at += counts[e]
        x, w = x8[token[rows_e]], W1[e].double()
        # (1.3e-5 of a row's products, below 2^-12 of their magnitudes)
        terms = 2.0 ** -12 * (x.abs() @ w.abs()) + 2.0 ** -20
        ref = x @ w + b1[e].double()
        H = a["H"][rows_e].view(torch.float8_e4m3fn).double()
        for h in (0, 1):
            s = torch.exp2(a["Hs"][rows_e][:, h * nb:(h + 1) * nb].double() - 127).repeat_interleave(128, 1)[:, :n]
            half = slice(h * n, (h + 1) * n)
            bad += _far_off(torch, H[:, half] * s, ref[:, half], terms[:, half])
    assert at == first and int(bad) == 0
