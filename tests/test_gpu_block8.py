"""The 8-bit operators on the GPU against the oracle in 64 bits.

Codes and scales of given values are a function of those values: they match exactly.  What is computed before it is
rounded (A, H) may land on the other side of a rounding step: its bound counts such steps.  The backward is compared on
the device's own kept values, with the tolerance of the 16-bit layer's tests (bf16 rows between its products).
"""
import numpy as np
import pytest

import oracle
from dense_reference import rel_err
from oracle import block8
from paper_2512_14080_amd import workloads as W
from test_gpu_parity import TOL, _torch, expert_biases, oracle_routing, oracle_scores

pytestmark = pytest.mark.gpu


def _bf16(x):
    torch = _torch()
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).cuda()


def _same(a, b):
    np.testing.assert_array_equal(np.isnan(a), np.isnan(b))
    np.testing.assert_array_equal(a[~np.isnan(a)], b[~np.isnan(b)])


# ------------------------------------------------------------------ the format
def _special_rows(rows, cols):
    """Rows of many magnitudes, and in the first ones zeros, subnormals, the largest values, infinities and NaN."""
    rng = np.random.default_rng(rows + cols)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-40, 40, (rows, 1)))
    for i, v in enumerate([0.0, 2.0 ** -133, 2.0 ** -126 * 1.5, 3.38e38, np.inf, np.nan, 448.0, 450.0, -0.0, -np.inf]):
        if i < rows:
            x[i, :: 3] = v
            if i < 4:
                x[i] = v
    return x


@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 128), (3, 136), (17, 1000), (64, 1024), (5, 4104), (1000, 640),
                                       (129, 392)])
def test_rows_through_the_format(rows, cols):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    X = _bf16(_special_rows(rows, cols))
    stride = B.scale_stride(cols)
    q = torch.full((rows + 1, cols), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((rows + 1, stride), 0xCD, dtype=torch.uint8, device="cuda")
    back = torch.full((rows + 1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    B.moe_quantize_rows(rows, cols, X, q, s)
    B.moe_dequantize_rows(rows, cols, q, s, back)
    torch.cuda.synchronize()
    codes, e, values = block8.quantize(X.double().cpu().numpy())
    got = q.cpu().numpy()
    nan = (codes & 0x7F) == 0x7F  # (either NaN code)
    np.testing.assert_array_equal((got[:rows] & 0x7F) == 0x7F, nan)
    np.testing.assert_array_equal(got[:rows][~nan], codes[~nan])
    scales = s.cpu().numpy()
    blocks = e.shape[1]
    np.testing.assert_array_equal(scales[:rows, :blocks], e + 127)
    assert (scales[:rows, blocks:] == 127).all()
    want = torch.from_numpy(values).to(torch.bfloat16).double().numpy()  # (rounds below 2^-133 only)
    _same(back[:rows].double().cpu().numpy(), want)
    # nothing past the rows
    assert (got[rows] == 0xAB).all() and (scales[rows] == 0xCD).all() and (back[rows] == 7.0).all()


@pytest.mark.parametrize("d,n,E", [(128, 64, 8), (256, 128, 8), (384, 192, 16), (128, 448, 8)])
def test_experts_through_the_format(d, n, E):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    rng = np.random.default_rng(n)
    W1 = rng.standard_normal((E, d, 2 * n)) * np.exp2(rng.integers(-8, 8, (E, 1, 1)))
    W2 = rng.standard_normal((E, n, d)) * 0.02
    W1[0, 3, 5], W1[1, :, :n], W2[2, n - 1, d - 1], W2[3] = np.inf, 0.0, np.nan, 0.0
    w1, w2 = _bf16(W1), _bf16(W2)
    D = B.dims(1, d, n, E, 1)
    qw = B.QExperts(D)
    qw.buf.fill_(0xAB)
    o1 = torch.full((E + 1, d, 2 * n), 7.0, dtype=torch.bfloat16, device="cuda")
    o2 = torch.full((E + 1, n, d), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.MoEError):
        B.moe_dequantize_experts(D, qw, o1, o2)
    B.moe_quantize_experts(D, w1, w2, qw)
    B.moe_dequantize_experts(D, qw, o1, o2)
    torch.cuda.synchronize()
    v1, v2 = block8.through_experts(w1.double().cpu().numpy(), w2.double().cpu().numpy())
    _same(o1[:E].double().cpu().numpy(), v1)
    _same(o2[:E].double().cpu().numpy(), v2)
    assert (o1[E] == 7.0).all() and (o2[E] == 7.0).all()


# ------------------------------------------------------------------ the layer
def _layer(cfg, held8, seed=0, mode=None, keep_x=False, biased=False, edit=None):
    _torch()
    from paper_2512_14080_amd.layer import DeviceLayer
    inp = W.make_inputs(cfg, seed)
    if edit is not None:
        edit(inp)
    _, S = oracle_scores(inp)
    b1, b2 = expert_biases(cfg, seed, 0.1) if biased else (None, None)
    layer = DeviceLayer(inp, round_mode=mode, scores_in=S, b1=b1, b2=b2, held8=held8, keep_x=keep_x)
    layer.ckpt.buf.fill_(0xAB)
    _, _, R = oracle_routing(S, cfg.K, mode, cfg.m_tile)
    return inp, R, layer, b1, b2


def _kept(layer):
    """The values that the checkpoint stands for, and its H codes."""
    a = {k: v.cpu().numpy() for k, v in layer.ckpt.arrays().items()}
    n, nb = layer.n, -(-layer.n // 128)

    def value(q, s):
        return block8.VALUES[q] * np.ldexp(1.0, np.repeat(s.astype(int) - 127, 128, 1)[:, :q.shape[1]])

    H = np.concatenate([value(a["H"][:, :n], a["Hs"][:, :nb]), value(a["H"][:, n:], a["Hs"][:, nb:2 * nb])], 1)
    X = value(a["X"], a["Xs"][:, :-(-layer.d // 128)]) if "X" in a else None
    return H, X, a


def _check_kept_h(H, ref, terms, off):
    """H: kept values; ref: the 64-bit H; terms: bound of the products' own error.  Rounding is monotone, so values y and x
    on a grid of steps s round to r(y), r(x) with |r(y) - r(x)| <= |y - x| + s: the products' error (up to 1.3e-5 of an
    H row's spread on the 8-bit matrix instruction, more than the smallest step of a block, 2^-9 / 224 of its largest
    value) and one step (2^-3 |value|, or the block's smallest).  At most a share `off` may differ at all."""
    want = block8.through_halves(ref)
    n = ref.shape[1] // 2
    e = np.concatenate([np.repeat(block8.exponents(h, (1, 128)), 128, 1)[:, :n] for h in (ref[:, :n], ref[:, n:])], 1)
    step = np.maximum(np.abs(want) / 8, np.ldexp(1.0, e - 9))
    assert (np.abs(H - want) <= terms + step * 1.0000001).all()
    assert (H != want).mean() <= off


def _magnitudes(X, W1, R):
    """sum |x| |w| of every H."""
    t = np.zeros((R.P, W1.shape[2]))
    for e in range(W1.shape[0]):
        a, b = int(R.offsets[e]), int(R.offsets[e + 1])
        t[a:b] = np.abs(X[R.row_token[a:b]]) @ np.abs(W1[e])
    return t


def _check_o(O, fw, R, W2q, rows_quantised):
    """2^-8 of each Y and of O (bf16 stores); the matrix instruction adds its products in about 2^-12 of their
    magnitudes' sum; and up to three codes of a row of A a step (2^-3) off."""
    A, Y = fw["A8"] if rows_quantised else fw["A"], fw["Y"]
    err = np.zeros_like(fw["O"])
    for e in range(W2q.shape[0]):
        a, b = int(R.offsets[e]), int(R.offsets[e + 1])
        if a == b:
            continue
        terms = np.abs(A[a:b]) @ np.abs(W2q[e])
        flip = np.stack([(np.abs(A[a:b]) * np.abs(W2q[e][:, c])[None]).max(1) for c in range(W2q.shape[2])], 1)
        row = 2.0 ** -8 * np.abs(Y[a:b]) + 2.0 ** -12 * terms + 3 / 8 * flip
        np.add.at(err, R.row_token[a:b], R.row_w[a:b, None] * row)
    assert (np.abs(O - fw["O"]) <= err + 2.0 ** -8 * np.abs(fw["O"]) + 1e-30).all()


def _check_backward(layer, inp, R, H, X, b2):
    torch = _torch()
    layer.backward()
    torch.cuda.synchronize()
    P = R.P
    W1, W2, Wr, dO = (inp.f32(k) for k in ("W1", "W2", "Wr", "dO"))
    bw = block8.backward_ckpt(dO, X, H, W1, W2, Wr, R, b2=b2)
    got = {"dX": layer.dX, "dW1": layer.dW1, "dW2": layer.dW2, "dWr": layer.dWr, "dbias": layer.dbias, "dS": layer.dS[:P]}
    if b2 is not None:
        got.update(db1=layer.db1, db2=layer.db2)
    errs = {k: rel_err(v.float().cpu().numpy(), bw[k]) for k, v in got.items()}
    print({k: f"{v:.2e}" for k, v in errs.items()}, flush=True)
    assert max(errs.values()) <= TOL, errs


def check_held(cfg, held8, seed=0, mode=None, keep_x=False, biased=False):
    torch = _torch()
    inp, R, layer, b1, b2 = _layer(cfg, held8, seed, mode, keep_x, biased)
    layer.route()
    layer.forward()
    torch.cuda.synchronize()
    X, W1, W2 = (inp.f32(k).astype(np.float64) for k in ("X", "W1", "W2"))
    H, Xk, raw = _kept(layer)
    P = R.P
    O = layer.O.double().cpu().numpy()
    if held8 == "quant":
        fw = block8.forward_quant(X, W1, W2, R, b1, b2)
        # (the 8-bit values are at most 1 + 2^-4 of the 16-bit ones)
        _check_kept_h(H[:P], fw["H"], 2.0 ** -12 * 1.13 * _magnitudes(X, W1, R), 1e-2)
        _check_o(O, fw, R, fw["W2q"], True)
    else:
        fw = oracle.forward(X, W1, W2, R, dtype=np.float64, b1=b1, b2=b2)
        _check_kept_h(H[:P], fw["H"], 2.0 ** -18 * _magnitudes(X, W1, R), 2e-3)
        assert rel_err(O, fw["O"]) <= TOL
    # rows behind the last expert's are left alone
    assert (raw["H"][P:] == 0xAB).all() and (raw["Hs"][P:] == 0xAB).all()
    if keep_x:
        np.testing.assert_array_equal(Xk, block8.through(X))
    _check_backward(layer, inp, R, H[:P], Xk if keep_x else X, b2)
    return layer, R


SHAPES = [
    W.MoEConfig("one", T=1, d=128, n=64, E=8, K=1, m_tile=16),          # one row; a half block of n
    W.MoEConfig("few", T=3, d=384, n=192, E=40, K=3, m_tile=16),        # mostly empty experts; one block and a half
    W.MoEConfig("all", T=70, d=256, n=128, E=8, K=8, m_tile=16),        # every expert holds every token
    W.MoEConfig("b320", T=129, d=640, n=320, E=16, K=4, m_tile=16),     # two blocks and a half
    W.MoEConfig("deep", T=300, d=1152, n=64, E=8, K=2, m_tile=32),      # k of nine blocks, n of a half
    W.MoEConfig("wide", T=700, d=256, n=640, E=8, K=2, m_tile=64),      # five blocks: 256-wide tiles with an uneven end
    W.MoEConfig("full", T=2100, d=512, n=256, E=8, K=2, m_tile=128),    # full 256-row tiles and partial ones
    W.MoEConfig("skew", T=500, d=256, n=128, E=64, K=4, m_tile=16, zipf_s=1.5),  # empty, tiny and hot experts
]


@pytest.mark.parametrize("cfg", SHAPES, ids=lambda c: c.name)
@pytest.mark.parametrize("held8", ["ckpt", "quant"])
def test_layer(cfg, held8):
    check_held(cfg, held8, seed=3)


@pytest.mark.parametrize("held8", ["ckpt", "quant"])
@pytest.mark.parametrize("mode", [None, "nearest", "up"])
def test_layer_with_everything(held8, mode):
    """Biases, X kept in 8 bits, and a rounded routing, whose capacity exceeds its rows."""
    check_held(W.MoEConfig("odd", T=1000, d=384, n=192, E=24, K=3, m_tile=32), held8, 4, mode, True, True)


def test_held_layers_full_rows_per_expert():
    """Many rows an expert at the narrow layer sizes: weight gradients in row chunks."""
    check_held(W.MoEConfig("long", T=5000, d=128, n=64, E=8, K=4, m_tile=128), "quant", 5, "nearest", True)


FORWARD = SHAPES + [
    W.MoEConfig("t10", T=10, d=896, n=320, E=8, K=8, m_tile=16),        # one row block of 10 rows, K = E
    W.MoEConfig("t16", T=16, d=768, n=256, E=8, K=8, m_tile=16),        # its last size
    W.MoEConfig("t17", T=17, d=768, n=256, E=8, K=8, m_tile=16),        # two row blocks
    W.MoEConfig("m20", T=20, d=256, n=128, E=16, K=16, m_tile=16),      # two at their largest mean
    W.MoEConfig("m21", T=21, d=256, n=128, E=16, K=16, m_tile=16),      # four
    W.MoEConfig("t128", T=128, d=640, n=192, E=8, K=4, m_tile=16),      # rows past one group of four
    W.MoEConfig("t150", T=150, d=256, n=64, E=120, K=8, m_tile=16, zipf_s=1.5),   # hot experts of many groups
    W.MoEConfig("t140", T=140, d=640, n=192, E=24, K=8, m_tile=16, zipf_s=3.0),
    W.MoEConfig("t5", T=5, d=1280, n=1152, E=8, K=3, m_tile=16),        # nine blocks of n, ten of d, on eight waves
]


@pytest.mark.parametrize("cfg", FORWARD, ids=lambda c: c.name)
@pytest.mark.parametrize("biased", [False, True])
def test_forward_without_a_checkpoint(cfg, biased):
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    inp, R, layer, b1, b2 = _layer(cfg, "quant", seed=10, biased=biased)
    layer.route()
    B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
    layer.ws_f.fill_(0xFF)  # NaN in every type: nothing unwritten is used
    B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, None, layer.O, layer.ws_f, eb=layer.eb)
    torch.cuda.synchronize()
    fw = block8.forward_quant(inp.f32("X"), inp.f32("W1"), inp.f32("W2"), R, b1, b2)
    _check_o(layer.O.double().cpu().numpy(), fw, R, fw["W2q"], True)
    assert (layer.ckpt.buf == 0xAB).all()


FEW = [
    (W.MoEConfig("k16", T=1, d=256, n=1152, E=32, K=16, m_tile=16), None),               # 144 steps on eight waves
    (W.MoEConfig("half", T=8, d=640, n=320, E=64, K=4, m_tile=16), None),                # E / 2 rows, an uneven n
    (W.MoEConfig("t32", T=32, d=128, n=64, E=64, K=1, m_tile=16), None),                 # one step a token
    (W.MoEConfig("t64", T=64, d=256, n=128, E=64, K=1, m_tile=16), None),                # E rows
    (W.MoEConfig("same", T=6, d=384, n=192, E=48, K=4, m_tile=16, zipf_s=3.0), None),    # tokens that share experts
    (W.MoEConfig("up", T=9, d=384, n=192, E=64, K=3, m_tile=8), "up"),                   # rounded: more rows than T K
    (W.MoEConfig("down", T=9, d=384, n=192, E=64, K=3, m_tile=8), "down"),               # and hardly any
]


@pytest.mark.parametrize("cfg,mode", FEW, ids=lambda c: getattr(c, "name", ""))
@pytest.mark.parametrize("biased", [False, True])
def test_few_tokens(cfg, mode, biased):
    """At most E / 2 rows, or E of few weights: by row and by token where they are a token choice's."""
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    inp, R, layer, b1, b2 = _layer(cfg, "quant", seed=21, mode=mode, biased=biased)
    layer.route()
    B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
    fw = block8.forward_quant(inp.f32("X"), inp.f32("W1"), inp.f32("W2"), R, b1, b2)
    out = []
    for _ in range(2):
        layer.ws_f.fill_(0xFF)
        layer.O.fill_(7.0)
        B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, None, layer.O, layer.ws_f, eb=layer.eb)
        out.append(layer.O.clone())
    torch.cuda.synchronize()
    assert torch.equal(*out)
    _check_o(out[0].double().cpu().numpy(), fw, R, fw["W2q"], True)


def test_decode_steps_in_a_graph():
    """Routing and the forward of few tokens, captured once and replayed on other tokens between eager calls."""
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    cfg = W.MoEConfig("decode", T=4, d=384, n=192, E=40, K=3, m_tile=16)
    _, _, layer, _, _ = _layer(cfg, "quant", seed=31, biased=True)
    B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
    layer.route_flags &= ~B.MOE_ROUTE_SCORES_IN

    def step():
        layer.route()
        B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, None, layer.O, layer.ws_f, eb=layer.eb)

    tokens = [torch.randn_like(layer.X) for _ in range(4)]
    want = []
    for x in tokens:
        layer.X.copy_(x)
        step()
        want.append(layer.O.clone())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for i in (2, 0, 3, 1, 1):
        layer.X.copy_(tokens[i])
        layer.O.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.O, want[i]), i
        step()
        assert torch.equal(layer.O, want[i]), i


def test_a_tokens_output_does_not_depend_on_its_tile():
    """Many rows behind a long n: whole rounds of tiles and a last one in quarters (282 to 298 tiles of 256 x 256, two per
    m-tile, the second of 128 columns), every token with the bits that it gets among few."""
    torch = _torch()
    from paper_2512_14080_amd import binding as B
    small = W.MoEConfig("few", T=450, d=384, n=4096, E=8, K=2, m_tile=16)
    big = W.MoEConfig("many", T=18000, d=384, n=4096, E=8, K=2, m_tile=16)

    def forward(layer):
        layer.route()
        layer.ws_f.fill_(0xFF)
        layer.O.fill_(7.0)
        B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, None, layer.O, layer.ws_f, eb=layer.eb)

    inp, R, few, b1, b2 = _layer(small, "quant", seed=12, biased=True)
    B.moe_quantize_experts(few.D, few.W1, few.W2, few.qw)
    forward(few)
    torch.cuda.synchronize()
    fw = block8.forward_quant(inp.f32("X"), inp.f32("W1"), inp.f32("W2"), R, b1, b2)
    _check_o(few.O.double().cpu().numpy(), fw, R, fw["W2q"], True)
    _, R, many, _, _ = _layer(big, "quant", seed=13, biased=True)
    tiles = 2 * -(-np.diff(R.offsets) // 256).sum()
    assert 256 < tiles <= 256 + 64, tiles
    many.qw, many.eb = few.qw, few.eb
    forward(many)
    for t in range(0, big.T, small.T):
        few.X.copy_(many.X[t:t + small.T])
        few.tc.arrays()["scores"].copy_(many.tc.arrays()["scores"][t:t + small.T])
        forward(few)
        assert torch.equal(few.O, many.O[t:t + small.T]), t


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("T,E", [(9, 16), (400, 16), (9, 64)])
def test_one_broken_token_stays_one(bad, T, E):
    """A value that is not finite reaches its own token's output only."""
    torch = _torch()
    from paper_2512_14080_amd import binding as B

    def edit(inp):
        inp.X[5, 17] = W.bf16_bits_from_f32(np.array([1.0], np.float32))[0]  # (the scores are the sound token's)

    cfg = W.MoEConfig("broken", T=T, d=256, n=128, E=E, K=2, m_tile=16)
    inp, R, layer, _, _ = _layer(cfg, "quant", seed=6, edit=edit)
    layer.route()
    sound = layer.X.clone()
    keep = torch.arange(T, device="cuda") != 5
    for ckpt in (layer.ckpt, None):
        out = []
        for value in (1.0, float(bad)):
            layer.X.copy_(sound)
            layer.X[5, 17] = value
            B.moe_quantize_experts(layer.D, layer.W1, layer.W2, layer.qw)
            B.moe_fwd_quant(layer.D, layer.X, layer.qw, layer.routing, ckpt, layer.O, layer.ws_f)
            torch.cuda.synchronize()
            out.append(layer.O.clone())
        assert torch.isnan(out[1][5]).any()
        assert torch.equal(out[1][keep], out[0][keep])


def test_steps_in_a_graph_and_on_another_stream():
    """A captured step (quantise, forward, backward) replayed between eager ones, on new inputs, and an eager step on a
    side stream: all as the eager step on the default stream."""
    torch = _torch()
    cfg = W.MoEConfig("graph", T=600, d=256, n=192, E=16, K=2, m_tile=64)
    for held8 in ("quant", "ckpt"):
        _, _, layer, _, _ = _layer(cfg, held8, seed=7, keep_x=True, biased=True)
        X0 = layer.X.clone()
        names = ("O", "dX", "dW1", "dW2", "dWr", "dbias", "db1", "db2")

        def result():
            torch.cuda.synchronize()
            return {k: getattr(layer, k).clone() for k in names}

        layer.route()

        def step(stream=None):
            layer.forward(stream)
            layer.backward(stream)

        want = []
        for k in range(3):
            layer.X.copy_(X0 * (k + 1))
            step()
            want.append(result())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        side = torch.cuda.Stream()
        for k in (2, 0, 1):
            layer.X.copy_(X0 * (k + 1))
            for t in ("O", "dX", "dW1", "dW2"):
                getattr(layer, t).fill_(3.0)
            g.replay()
            got = result()
            assert all(torch.equal(got[n], want[k][n]) for n in names), (held8, k)
            side.wait_stream(torch.cuda.current_stream())
            step(side)
            got = result()
            assert all(torch.equal(got[n], want[k][n]) for n in names), (held8, k)


def test_two_layers_at_once():
    """Two layers with buffers of their own on two streams."""
    torch = _torch()
    cfg = W.MoEConfig("two", T=900, d=384, n=128, E=16, K=4, m_tile=64)
    layers = [_layer(cfg, "quant", seed=s)[2] for s in (8, 9)]
    want = []
    for l in layers:
        l.step()
        torch.cuda.synchronize()
        want.append([l.O.clone(), l.dX.clone(), l.dW1.clone()])
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(4):
        for l, s in zip(layers, streams):
            l.step(s)
    torch.cuda.synchronize()
    for l, w in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip((l.O, l.dX, l.dW1), w))
