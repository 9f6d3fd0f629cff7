"""What the 8-bit forward may be off by, tighter than element by element: the codes that A is held in, exactly, those of a
kept H all but a few, and O's error in the root mean square."""
import numpy as np
import pytest

import oracle
from dense_reference import rel_fro
from oracle import block8
from paper_2512_14080_amd import workloads as W
from test_block8_cpu import built
from test_block8_launches import _names, launches
from test_gpu_parity import _torch, expert_biases, oracle_routing, oracle_scores

# (dims with K = 1, what computes A without and with a checkpoint)
PATHS = [
    ((1, 256, 192, 8, 1), "stream8_row_up", "Li128ELi256E"),
    ((16, 256, 256, 8, 1), "stream8_gemm", "Li128ELi256E"),       # groups of 16 rows
    ((40, 384, 320, 16, 1), "stream8_gemm", "Li128ELi256E"),      # of 32
    ((700, 384, 192, 8, 1), "Li128ELi256E", "Li128ELi256E"),
    ((3000, 512, 448, 8, 1), "Li256ELi256E", "Li256ELi256E"),
    ((100000, 512, 128, 8, 1), "Li256ELi256E", "Li256ELi256E"),   # several tiles a workgroup, 256-wide both
]


@built
@pytest.mark.parametrize("dims,plain,kept", PATHS)
def test_paths_of_the_cases(tmp_path, dims, plain, kept):
    for l, want in zip(launches([(dims, "quant", 0, False), (dims, "kept", 0, False)], tmp_path), (plain, kept)):
        assert want in _names([x for x in l if "OpUp8" in x[0] or "stream8" in x[0]][:1])


def _exact_inputs(dims, seed):
    """Inputs whose products are exact, and their A [T, n]: a token is one value v at one column, so H is one product;
    the gate is at least 112, where SiLU is the identity in fp32; A = 448 v^2 u has 15 bits.  The up weights are all codes of
    the type, so a block's A reach down to where a code of the next larger scale would lose bits."""
    T, d, n, E, _ = dims
    rng = np.random.default_rng(seed)
    v, at, e = rng.integers(8, 16, T) / 32, rng.integers(0, d, T), rng.integers(0, E, T)
    codes = block8.VALUES[np.r_[0:0x7F, 0x80:0xFF]]
    up = codes[rng.integers(0, codes.size, (E, d, n))]
    X, W1, W2 = np.zeros((T, d)), np.empty((E, d, 2 * n)), np.zeros((E, n, d))
    X[np.arange(T), at] = v
    W1[:, :, :n], W1[:, :, n:] = 448.0, up
    W2[:, np.arange(n), np.arange(n)] = 1.0  # so O is A as held
    scores = np.full((T, E), 0.25 / E, np.float32)
    scores[np.arange(T), e] = 0.75
    return X, W1, W2, scores, 448.0 * v[:, None] ** 2 * up[e, at]


@pytest.mark.gpu
@pytest.mark.parametrize("dims,plain,kept", PATHS)
def test_codes_of_a(dims, plain, kept):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    T, d, n, E, K = dims
    X, W1, W2, scores, A = _exact_inputs(dims, T)
    want = block8.through(A)
    # (the test sees a scale of twice the size)
    e = np.repeat(block8.exponents(A, (1, 128)), 128, 1)[:, :n]
    s = np.ldexp(1.0, e + 1)
    assert (block8.VALUES[block8.encode(A / s)] * s != want).any()

    def dev(x):
        return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).cuda()

    D = B.dims(*dims)
    r = B.Routing(D, T)
    r.arrays()["scores"].copy_(torch.from_numpy(scores))
    B.moe_route(D, None, None, None, B.MOE_ROUTE_SCORES_IN, r)
    assert (r.arrays()["row_w"] == 1).all()
    qw = B.QExperts(D)
    B.moe_quantize_experts(D, dev(W1), dev(W2), qw)
    ws = torch.empty(B.moe_workspace_bytes(D, T, B.MOE_WS_FWD_QUANT), dtype=torch.uint8, device="cuda")
    for ckpt in (None, B.Checkpoint(D, T, keep_x=True)):
        ws.fill_(0xFF)
        O = torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_fwd_quant(D, dev(X), qw, r, ckpt, O, ws)
        O = O.double().cpu().numpy()
        np.testing.assert_array_equal(O[:, :n], want)
        assert (O[:, n:] == 0).all()


# The root mean square of O's error.  A rounding to bf16 is off by at most 2^-8 of its value, uniformly up to there at the
# worst: 2^-8 / sqrt 3.  O takes one, Y one more in the tiled projections.  The 8-bit instruction is 1.3e-5 of a row's spread
# off in H, which moves A by some 5e-5 of its value and so the share 5e-5 / 2^-4 of its codes, at the most, a step of up to
# 2^-3; few rows multiply the codes in bf16, where none moves.
ROUND = 2.0 ** -8 / 3 ** 0.5
MOVED = (5e-5 * 16) ** 0.5 / 8
OFF = {"few": ROUND, "stream": (ROUND ** 2 + MOVED ** 2) ** 0.5, "tiled": (2 * ROUND ** 2 + MOVED ** 2) ** 0.5,
       "kept": 2 ** 0.5 * ROUND}  # (H and so A from fp32 sums)


@pytest.mark.gpu
@pytest.mark.parametrize("cfg,path", [
    (W.MoEConfig("t1", T=1, d=1536, n=256, E=64, K=8, m_tile=16), "few"),
    (W.MoEConfig("t8", T=8, d=768, n=320, E=16, K=4, m_tile=16), "few"),
    (W.MoEConfig("t64", T=64, d=1024, n=256, E=64, K=8, m_tile=16), "stream"),
    (W.MoEConfig("t200", T=200, d=640, n=192, E=16, K=4, m_tile=16), "tiled"),
    (W.MoEConfig("t2000", T=2000, d=512, n=448, E=8, K=2, m_tile=16), "tiled"),
], ids=lambda x: getattr(x, "name", x))
@pytest.mark.parametrize("biased", [False, True])
def test_relative_error_of_o(cfg, path, biased):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    from paper_2512_14080_amd.layer import DeviceLayer
    inp = W.make_inputs(cfg, 5)
    _, S = oracle_scores(inp)
    b1, b2 = expert_biases(cfg, 5, 0.1) if biased else (None, None)
    layer = DeviceLayer(inp, scores_in=S, b1=b1, b2=b2, held8="quant")
    layer.route()
    B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
    _, _, R = oracle_routing(S, cfg.K, None, cfg.m_tile)
    ref = block8.forward_quant(inp.f32("X"), inp.f32("W1"), inp.f32("W2"), R, b1, b2)["O"]
    for ckpt, bound in ((None, OFF[path]), (layer.ckpt, OFF["kept"])):
        B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, ckpt, layer.O, layer.ws_f, eb=layer.eb)
        err = rel_fro(layer.O.double().cpu().numpy(), ref)
        print(cfg.name, path, f"{err:.2e} of {bound:.2e}", flush=True)
        assert err <= bound


@pytest.mark.gpu
@pytest.mark.parametrize("dims", [(4096, 1024, 256, 64, 8), (2000, 512, 192, 8, 2), (500, 1536, 320, 16, 2)])
def test_codes_of_a_kept_h(dims):
    """fp32 sums are some 2^-21 of a row's spread off.  A border between two codes lies every 2^-4 to 2^-3 of a value, so the
    share of values that one lies next to is at most 2^-21 * 16 * E[spread / |value|], with 3 for the mean: 2.3e-5."""
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    T, d, n, E, K = dims
    D = B.dims(*dims)
    g = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    X, W1, W2 = normal(T, d), normal(E, d, 2 * n, std=0.02), normal(E, n, d, std=0.02)
    r = B.Routing(D, T * K)
    r.arrays()["scores"].copy_(torch.softmax(torch.randn((T, E), generator=g, device="cuda"), 1))
    B.moe_route(D, None, None, None, B.MOE_ROUTE_SCORES_IN, r)
    qw, ckpt = B.QExperts(D), B.Checkpoint(D, r.capacity, keep_x=True)
    B.moe_quantize_experts(D, W1, W2, qw)
    B.moe_dequantize_experts(D, qw, W1, W2)  # the values that the codes stand for
    ws = torch.empty(B.moe_workspace_bytes(D, r.capacity, B.MOE_WS_FWD_QUANT), dtype=torch.uint8, device="cuda")
    B.moe_fwd_quant(D, X, qw, r, ckpt, torch.empty_like(X), ws)
    a, nb, x8 = ckpt.arrays(), -(-n // 128), torch.empty_like(X)
    B.moe_dequantize_rows(T, d, a["X"], a["Xs"], x8)
    offsets, token = r.arrays()["offsets"].tolist(), r.arrays()["row_token"].long()
    off = 0
    for e in range(E):
        rows = slice(offsets[e], offsets[e + 1])
        H = x8[token[rows]].double() @ W1[e].double()
        for h in (0, 1):
            s = torch.exp2(a["Hs"][rows][:, h * nb:(h + 1) * nb].double() - 127).repeat_interleave(128, 1)[:, :n]
            v = H[:, h * n:(h + 1) * n] / s
            step = torch.exp2(torch.frexp(v)[1].clamp_min(-5).double() - 4)
            got = a["H"][rows][:, h * n:(h + 1) * n].view(torch.float8_e4m3fn).double()
            off += int((got != (v / step).round() * step).sum())
    share = off / (2 * n * offsets[E])
    print(f"{share:.1e} of the codes", flush=True)
    assert share <= 2.0 ** -21 * 16 * 3
