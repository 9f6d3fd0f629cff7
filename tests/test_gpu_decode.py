"""moe_decode and moe_decode_quant on the GPU against their definition in 64 bits (dense_bounds), by element."""
import numpy as np
import pytest

import dense_bounds as DB
from oracle import block8

pytestmark = pytest.mark.gpu


def _t():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _inputs(T, d, n, E, K, seed, biases=False, residual=True):
    """Tokens whose K + 1 best logits are apart (the rounding of fp32 sums must not choose), weights, biases."""
    torch = _t()
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    Wr, W1, W2 = normal((d, E), d ** -0.5), normal((E, d, 2 * n), 0.05), normal((E, n, d), 0.05)
    bias, b1, b2 = (normal(s, 0.1, torch.float32) if biases else None for s in ((E,), (E, 2 * n), (E, d)))
    X = normal((3 * T + 16, d), 1.0)
    l = X.double() @ Wr.double() + (0 if bias is None else bias.double())
    v = torch.sort(l, dim=1, descending=True).values[:, :K + 1]
    apart = (v[:, :-1] - v[:, 1:]).amin(1) > 2 ** -11 if v.shape[1] > 1 else torch.ones(len(X), dtype=torch.bool, device="cuda")
    X = X[apart][:T].contiguous()
    assert X.shape[0] == T
    R = normal((T, d), 1.0) if residual else None
    return X, Wr, bias, W1, W2, b1, b2, R


class Call:
    """The call's buffers, each with a guard behind it."""

    def __init__(self, T, d, n, E, K, quant=False):
        torch = _t()
        from paper_2512_14080_amd import binding as B
        self.B, self.D, self.T, self.d, self.K = B, B.dims(T, d, n, E, K), T, d, K
        self.quant = quant
        self.O = torch.full((T * d + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        self.idx = torch.full((T * K + 16,), -5, dtype=torch.int32, device="cuda")
        self.w = torch.full((T * K + 16,), -5.0, device="cuda")
        self.need = B.moe_workspace_bytes(self.D, 0, B.MOE_WS_DECODE_QUANT if quant else B.MOE_WS_DECODE)
        self.buf = torch.full((self.need + 512,), 0x7F, dtype=torch.uint8, device="cuda")  # (counters, sums: all garbage)
        self.off = (-self.buf.data_ptr()) % 256
        self.ws = self.buf[self.off:self.off + self.need]

    def __call__(self, X, Wr, bias, W1, W2, b1, b2, R, q=None, stream=None, O=None):
        eb = self.B.expert_bias(b1, b2)
        O = self.O if O is None else O
        if self.quant:
            self.B.moe_decode_quant(self.D, X, Wr, bias, q, R, O, self.ws, self.idx, self.w, stream, eb=eb)
        else:
            self.B.moe_decode(self.D, X, Wr, bias, W1, W2, R, O, self.ws, self.idx, self.w, stream, eb=eb)

    def results(self):
        torch = _t()
        torch.cuda.synchronize()
        n, k = self.T * self.d, self.T * self.K
        assert bool((self.O[n:] == 7.0).all()) and bool((self.idx[k:] == -5).all()) and bool((self.w[k:] == -5.0).all())
        assert bool((self.buf[self.off + self.need:] == 0x7F).all())
        return self.O[:n].view(self.T, self.d).clone(), self.idx[:k].view(self.T, self.K).clone(), self.w[:k].view(self.T, self.K).clone()


SHAPES = [
    # T, d, n, E, K, biases, residual
    (1, 128, 64, 8, 1, False, False),        # the smallest
    (1, 1536, 256, 128, 8, False, True),     # by token, k sliced
    (1, 256, 64, 8, 8, True, True),          # every expert
    (1, 384, 1088, 16, 16, True, False),     # by token, A through memory (K n > 8192)
    (2, 640, 192, 64, 6, True, True),
    (3, 512, 320, 200, 10, False, True),     # four values of a lane in the selection
    (4, 1024, 64, 128, 16, True, True),
    (5, 896, 192, 40, 3, False, True),       # by group from here on
    (7, 1024, 256, 64, 8, True, True),
    (8, 128, 64, 8, 8, True, True),          # eight rows for every expert
    (9, 256, 128, 1024, 2, True, True),      # selection as items, 16 values of a lane
    (16, 768, 1024, 32, 2, False, True),
    (17, 640, 448, 8, 2, True, True),        # two row blocks
    (31, 256, 64, 512, 16, False, True),     # eight values of a lane
    (33, 384, 64, 8, 8, True, True),         # 33 rows in a group: two passes of two row blocks
    (64, 256, 128, 128, 8, True, True),      # one row block
    (64, 384, 64, 8, 8, False, False),       # 64 rows in every group
    (64, 128, 192, 1024, 16, True, True),    # the largest lists
    (23, 1280, 64, 24, 1, False, True),      # K = 1
]


@pytest.mark.parametrize("T,d,n,E,K,biases,residual", SHAPES)
def test_decode(T, d, n, E, K, biases, residual):
    torch = _t()
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, d, n, E, K, 100 + T + d, biases, residual)
    idx, w, ew, gap = DB.select(X, Wr, bias, K)
    assert gap > 2 ** -12
    ref, bound = DB.decode(X, W1, W2, b1, b2, R, idx, w, ew)
    call = Call(T, d, n, E, K)
    call(X, Wr, bias, W1, W2, b1, b2, R)
    O, gi, gw = call.results()
    assert torch.equal(gi.long(), idx)
    DB.within(gw, w, ew, "weights")
    print("share of the bound:", DB.within(O, ref, bound, "O"), flush=True)
    # the same again, on used buffers: every sum has its order
    call(X, Wr, bias, W1, W2, b1, b2, R)
    again = call.results()
    assert all(torch.equal(a, b) for a, b in zip(again, (O, gi, gw)))


@pytest.mark.parametrize("T", [1, 6, 40])
def test_decode_without_outputs_and_in_place(T):
    """No selection asked for, R added in place, another stream."""
    torch = _t()
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, 256, 128, 32, 4, 5)
    call = Call(T, 256, 128, 32, 4)
    call(X, Wr, bias, W1, W2, b1, b2, R)
    O, _, _ = call.results()
    B = call.B
    out = R.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.moe_decode(call.D, X, Wr, bias, W1, W2, out, out, call.ws, stream=side)
    side.synchronize()
    assert torch.equal(out, O)


def test_ties_go_to_the_lower_expert():
    """Columns of W_r alike give scores alike, bit for bit."""
    torch = _t()
    for T, E, K in ((1, 128, 8), (5, 64, 6), (20, 256, 16)):
        X, Wr, _, W1, W2, b1, b2, R = _inputs(T, 256, 64, E, K, 9)
        Wr = Wr[:, :E // 4].repeat(1, 4).contiguous()
        call = Call(T, 256, 64, E, K)
        call(X, Wr, None, W1, W2, b1, b2, R)
        _, gi, gw = call.results()
        l = (X.double() @ Wr[:, :E // 4].double()).repeat(1, 4)
        idx = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :K]
        assert torch.equal(gi.long(), idx)
        assert torch.equal(gw[:, 0], gw[:, 1])


@pytest.mark.parametrize("T", [1, 3, 7, 24, 64])
def test_selection_is_the_routing_calls(T):
    """topk_idx as moe_route writes it; topk_w up to the order of sums."""
    torch = _t()
    d, n, E, K = 512, 64, 96, 8
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, d, n, E, K, 21, True)
    call = Call(T, d, n, E, K)
    call(X, Wr, bias, W1, W2, b1, b2, R)
    _, gi, gw = call.results()
    r = call.B.Routing(call.D, T * K)
    call.B.moe_route(call.D, X, Wr, bias, 0, r)
    torch.cuda.synchronize()
    a = r.arrays()
    assert torch.equal(gi, a["topk_idx"])
    _, w, ew, _ = DB.select(X, Wr, bias, K)
    DB.within(gw, a["topk_w"].double(), 2 * ew)


@pytest.mark.parametrize("T", [2, 7, 24])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_token_that_is_not_finite_stays_alone(T, value):
    torch = _t()
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, 256, 64, 32, 4, 31)
    call = Call(T, 256, 64, 32, 4)
    call(X, Wr, bias, W1, W2, b1, b2, R)
    O, gi, _ = call.results()
    X2 = X.clone()
    X2[1, 5] = value
    call(X2, Wr, bias, W1, W2, b1, b2, R)
    O2, gi2, _ = call.results()
    rest = torch.arange(T) != 1
    assert torch.equal(O2[rest], O[rest]) and torch.equal(gi2[rest], gi[rest])
    assert bool(torch.isnan(O2[1]).any())
    sel = sorted(gi2[1].tolist())
    assert len(set(sel)) == 4 and sel[0] >= 0 and sel[-1] < 32  # (experts all the same)


def test_bias_of_minus_infinity_and_lowest_masks_experts():
    torch = _t()
    T, E, K = 12, 64, 6
    X, Wr, _, W1, W2, b1, b2, R = _inputs(T, 256, 64, E, K, 41)
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        bias = torch.zeros(E, device="cuda")
        bias[::2] = low
        # (masked experts' weights must not matter)
        W1m, W2m = W1.clone(), W2.clone()
        W1m[::2], W2m[::2] = float("nan"), float("inf")
        call = Call(T, 256, 64, E, K)
        call(X, Wr, bias, W1m, W2m, b1, b2, R)
        O, gi, gw = call.results()
        l = X.double() @ Wr.double()
        l[:, ::2] = -float("inf")
        v, idx = torch.sort(l, dim=1, descending=True, stable=True)
        w = torch.softmax(v[:, :K], 1)
        assert torch.equal(gi.long(), idx[:, :K])
        ew = w * (2 * DB.E(256) * (X.double().abs() @ Wr.double().abs()).amax(1, keepdim=True) + DB.F)
        DB.within(gw, w, ew)
        ref, bound = DB.decode(X, W1, W2, b1, b2, R, idx[:, :K], w, ew)
        DB.within(O, ref, bound)
    # nothing left: as many experts as asked for, outputs that are not numbers
    call(X, Wr, torch.full((E,), -float("inf"), device="cuda"), W1, W2, b1, b2, R)
    O, gi, _ = call.results()
    assert all(len(set(r)) == K and 0 <= min(r) and max(r) < E for r in gi.tolist())
    assert bool(torch.isnan(O).all())


@pytest.mark.parametrize("quant", [False, True])
def test_graphs_that_share_a_workspace(quant):
    """Two captured calls of different sizes on one workspace, replayed in turn between eager work, on changing inputs."""
    torch = _t()
    from paper_2512_14080_amd import binding as B
    calls, ins, qs = [], [], []
    for T in (1, 20):
        calls.append(Call(T, 256, 128, 32, 4, quant))
        ins.append(list(_inputs(T, 256, 128, 32, 4, 51 + T)))
        q = None
        if quant:
            q = B.QExperts(calls[-1].D)
            B.moe_quantize_experts(calls[-1].D, ins[-1][3], ins[-1][4], q)
        qs.append(q)
    ws = max((c.ws for c in calls), key=lambda t: t.numel())
    for c in calls:
        c.ws = ws
    graphs = []
    for c, i, q in zip(calls, ins, qs):
        c(*i, q=q)  # (the code is loaded before a capture)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c(*i, q=q)
        graphs.append(g)
    for rep in range(4):
        fresh = [_inputs(c.T, 256, 128, 32, 4, 200 + 10 * rep + c.T)[0] for c in calls]
        for c, i, x in zip(calls, ins, fresh):
            i[0].copy_(x)
            c.O.fill_(7.0)
        for g in graphs:
            g.replay()
        got = [c.results()[0] for c in calls]
        for c, i, q, o in zip(calls, ins, qs, got):
            c(*i, q=q)
            assert torch.equal(c.results()[0], o), rep


def test_calls_at_once_on_streams_of_their_own():
    """Calls under way together, each with its workspace: as alone."""
    torch = _t()
    from paper_2512_14080_amd import binding as B
    work = []
    for T, d, n, E, K, quant in ((1, 1536, 256, 128, 8, False), (7, 1024, 256, 64, 8, False), (40, 512, 192, 32, 4, False),
                                 (16, 1536, 256, 128, 8, True)):
        x = _inputs(T, d, n, E, K, 400 + T)
        call, q = Call(T, d, n, E, K, quant), None
        if quant:
            q = B.QExperts(call.D)
            B.moe_quantize_experts(call.D, x[3], x[4], q)
        call(*x, q=q)
        alone = call.results()
        work.append((call, x, q, alone, torch.cuda.Stream()))
    for rep in range(3):
        for call, *_ in work:
            call.O[:call.T * call.d].fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(10):
            for call, x, q, _, side in work:
                call(*x, q=q, stream=side)
        torch.cuda.synchronize()
        for call, _, _, alone, _ in work:
            assert all(torch.equal(a, b) for a, b in zip(call.results(), alone)), (rep, call.T)


QUANT = [(1, 1536, 256, 128, 8, False), (1, 128, 64, 8, 2, True), (2, 256, 1088, 16, 16, True), (3, 512, 192, 16, 4, True),
         (9, 896, 192, 40, 3, True), (16, 256, 128, 8, 4, False), (20, 1280, 64, 128, 2, True), (33, 384, 320, 8, 8, False),
         (64, 256, 128, 64, 8, True), (64, 256, 192, 512, 4, True), (48, 128, 960, 8, 6, False), (24, 512, 576, 16, 4, True)]


@pytest.mark.parametrize("T,d,n,E,K,biases", QUANT)
def test_decode_quant(T, d, n, E, K, biases):
    """Against the definition: X, A and the weights through the block format.  The kernels' sums move some codes of A to the
    other side of a step of up to 2^-4 of the value; such a code is off by what 1.3e-5 of H is among the values between
    two codes: 3 in 10^4 of them, 2^-4 (3e-4)^0.5 = 1.1e-3 of A's norm.  O's own rounding is at most 2^-8 = 3.9e-3."""
    torch = _t()
    from paper_2512_14080_amd import binding as B
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, d, n, E, K, 300 + T + d, biases)
    call = Call(T, d, n, E, K, quant=True)
    q = B.QExperts(call.D)
    B.moe_quantize_experts(call.D, W1, W2, q)
    call(X, Wr, bias, W1, W2, b1, b2, R, q=q)
    O, gi, gw = call.results()
    idx, w, ew, gap = DB.select(X, Wr, bias, K)
    assert gap > 2 ** -12 and torch.equal(gi.long(), idx)
    DB.within(gw, w, ew)
    x8 = torch.from_numpy(block8.through(X.double().cpu().numpy())).cuda()
    ref = R.double().clone()
    for e in torch.unique(idx).tolist():
        t, j = (idx == e).nonzero(as_tuple=True)
        w1 = torch.from_numpy(block8.through_halves(W1[e].double().cpu().numpy(), (128, 128))).cuda()
        w2 = torch.from_numpy(block8.through(W2[e].double().cpu().numpy(), (128, 128))).cuda()
        h = x8[t] @ w1 + (0 if b1 is None else b1[e].double())
        a = torch.nn.functional.silu(h[:, :n]) * h[:, n:]
        a = torch.from_numpy(block8.through(a.cpu().numpy())).cuda()
        y = a @ w2 + (0 if b2 is None else b2[e].double())
        ref.index_add_(0, t, w[t, j][:, None] * y)
    err = ((O.double() - ref).norm() / ref.norm()).item()
    print("O off by", err, flush=True)
    assert err <= 3.9e-3 + 1.1e-3
    call(X, Wr, bias, W1, W2, b1, b2, R, q=q)
    assert torch.equal(call.results()[0], O)


def test_layer_decode_is_route_and_forward():
    """DeviceLayer.decode against its route and forward, 16-bit and 8-bit."""
    torch = _t()
    from paper_2512_14080_amd import workloads as W
    from paper_2512_14080_amd.layer import DeviceLayer
    cfg = W.MoEConfig("decode", T=12, d=256, n=128, E=16, K=2, m_tile=64)
    for held8 in (None, "quant"):
        layer = DeviceLayer(W.make_inputs(cfg, 3), held8=held8)
        layer.step()
        torch.cuda.synchronize()
        O = layer.O.double()
        R = torch.zeros_like(layer.O)
        layer.decode(R)
        torch.cuda.synchronize()
        # each is within a few roundings of the same value: A's and O's (2^-8 each, by norm less), or the codes' steps
        err = ((layer.O.double() - O).norm() / O.norm()).item()
        print(held8, err, flush=True)
        assert err <= 2 * (3.9e-3 + (1.1e-3 if held8 else 3.9e-3))
    with pytest.raises(ValueError):
        DeviceLayer(W.make_inputs(cfg, 3), round_mode="nearest").decode()
    assert np.isfinite(layer.O.float().cpu().numpy()).all()
