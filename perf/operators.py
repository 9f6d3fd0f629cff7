"""Timing cases of the layer's 8-bit operators, with their plain forms.

Kinds of case:
  rows     moe_quantize_rows + moe_dequantize_rows: activations into 8-bit blocks of 128 and back
  experts  moe_quantize_experts + moe_dequantize_experts: the expert weights, blocks of 128 x 128
  serve    moe_fwd_quant: the forward with 8-bit expert products, on weights quantised once
  ckpt     moe_fwd_ckpt + moe_bwd_ckpt: a training step in 16 bits whose cached activations are held in 8
  quant    moe_quantize_experts + moe_fwd_quant + moe_bwd_ckpt: a training step with the 8-bit forward

The routing (which rows an expert has, and their weights) is the plan that a program has in hand: prepare() builds it.

The format: a block's scale is the least power of two 2^e (e >= -126) with every finite |x| <= 448 * 2^e, kept as the
byte e + 127; its codes are e4m3(x / 2^e), to nearest even.
"""
import math

import torch

own = False

_BF16, _F32, _F64, _E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn


def _layer(name, kind, T, d, n, E, K, m_tile=0, zipf=0.0, biases=False, keep_x=False):
    """m_tile: tile of the token rounding (to the nearest), 0 for token choice.  zipf: exponent of the router's skew.
    keep_x: X is kept in 8 bits too, and the backward pass reads that."""
    c = {"kind": kind, "T": T, "d": d, "n": n, "E": E, "K": K, "m_tile": m_tile, "zipf": zipf, "biases": biases,
         "keep_x": keep_x}
    return {"name": name, **c} if name else c


def _rows(name, rows, cols):
    c = {"kind": "rows", "rows": rows, "cols": cols}
    return {"name": name, **c} if name else c


def _experts(name, d, n, E):
    c = {"kind": "experts", "d": d, "n": n, "E": E}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the activations of a decode batch on the 1B-shaped layer: latency
        _rows("rows-1b-t64", 64, 1024),
        # a full microbatch of the 7B-shaped layer: bandwidth
        _rows("rows-7b", 32768, 1536),
        # a layer off the tuned grid (n an odd multiple of 64): a half block at the end of every expert
        _experts("experts-odd", 896, 192, 40),
        # the 7B-shaped layer's weights: a checkpoint being loaded, or the step after an optimiser's
        _experts("experts-7b", 1536, 256, 128),
        # one token through the 7B-shaped layer: a single user's decode step
        _layer("serve-7b-t1", "serve", 1, 1536, 256, 128, 8),
        # a decode batch of 64 on the 1B-shaped layer: nearly every expert has a few rows
        _layer("serve-1b-t64", "serve", 64, 1024, 256, 64, 8),
        # a large decode batch on a 30B-shaped layer: 0.8 GB of expert weights
        _layer("serve-30b-t256", "serve", 256, 4096, 512, 128, 8),
        # one prompt of odd length on the 7B size at the middle granularity, with biases: about 110 rows an expert
        _layer("prefill-7b-t1777", "serve", 1777, 1536, 512, 64, 4, biases=True),
        # a prefill batch on the coarse-grained layer (8 experts of n = 14336): the largest products
        _layer("prefill-coarse-t4096", "serve", 4096, 4096, 14336, 8, 2),
        # a training step off the tuned grid with everything on: biases, rounding to 64, X kept in 8 bits too
        _layer("ckpt-odd-t5003", "ckpt", 5003, 896, 192, 40, 3, m_tile=64, zipf=0.3, biases=True, keep_x=True),
        # the 7B-shaped layer's full microbatch with token rounding: the headline step, H kept in 8 bits
        _layer("ckpt-7b-tr", "ckpt", 32768, 1536, 256, 128, 8, m_tile=128),
        # the 1B-shaped layer's full microbatch with the 8-bit forward
        _layer("quant-1b-t16384", "quant", 16384, 1024, 256, 64, 8, keep_x=True),
    ]


# (d, n, E, K) of the repository's layer shapes
_SHAPES = [(1024, 256, 64, 8), (1536, 256, 128, 8), (2048, 128, 256, 8), (4096, 14336, 8, 2), (768, 256, 128, 8),
           (768, 512, 64, 4), (768, 1024, 32, 2), (1536, 512, 64, 4), (1536, 1024, 32, 2), (4096, 256, 256, 16),
           (4096, 512, 128, 8), (4096, 1024, 64, 4), (1536, 256, 512, 8), (1536, 1024, 16, 2)]
_COST_OPS, _COST_BYTES = 2.8e12, 2.3e9  # at most the largest listed cases'


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choices(["rows", "experts", "serve", "ckpt", "quant"], [2, 1, 6, 4, 2])[0]
        if kind == "rows":
            c = _rows("", _log_int(rng, 1, 65536), 8 * _log_int(rng, 16, 512))
            if c["rows"] * c["cols"] <= 32768 * 1536:
                return c
            continue
        if rng.random() < 0.5:
            d, n, E, K = rng.choice(_SHAPES)
        else:
            d = 128 * rng.randint(2, 32)
            n = 64 * _log_int(rng, 1, 24)
            E = 8 * _log_int(rng, 1, 32)
            K = min(rng.choice([1, 2, 3, 4, 6, 8, 8, 10, 16]), E // 2)
        if kind == "experts":
            c = _experts("", d, n, E)
        elif kind == "serve":
            c = _layer("", kind, _log_int(rng, 1, 8192), d, n, E, K, zipf=rng.choice([0.0, 0.0, 0.3]),
                       biases=rng.random() < 0.25)
        else:
            m_tile = rng.choice([0, 0, 64, 128, 128])
            c = _layer("", kind, _log_int(rng, 256, 32768), d, n, E, K, m_tile, rng.choice([0.0, 0.0, 0.3]),
                       rng.random() < 0.25, rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= _COST_OPS and w["bytes"] <= _COST_BYTES:
            return c


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    """Activations of a normalised residual stream (unit variance, a few channels large), weights of standard deviation
    0.02, a router whose logits have unit variance, gradients of unit variance."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype=_BF16):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)

    def activations(rows, cols):
        x = normal((rows, cols), 1.0)
        large = torch.randperm(cols, generator=g, device="cuda")[:max(1, cols // 256)]
        x[:, large] *= 8
        return x

    s = {}
    if case["kind"] == "rows":
        s["X"] = activations(case["rows"], case["cols"])
        return s
    d, n, E = case["d"], case["n"], case["E"]
    s["W1"] = normal((E, d, 2 * n), 0.02)
    s["W2"] = normal((E, n, d), 0.02)
    if case["kind"] == "experts":
        return s
    T, K, M = case["T"], case["K"], case["m_tile"]
    s["X"] = activations(T, d)
    s["Wr"] = normal((d, E), d ** -0.5)
    s["b1"] = s["b2"] = None
    if case["biases"]:
        s["b1"] = normal((E, 2 * n), 0.1, _F32)
        s["b2"] = normal((E, d), 0.1, _F32)
    if case["kind"] != "serve":
        s["dO"] = normal((T, d), 1.0)
    # the router's scores, and the selection: the K best, the lowest expert first among equals; then, with M, every
    # expert's count rounded to the nearest multiple of M (a tie down), its lowest tokens dropped or best others added
    logits = s["X"].to(_F32) @ s["Wr"].to(_F32)
    if case["zipf"]:
        logits -= case["zipf"] * (torch.randperm(E, generator=g, device="cuda") + 1).to(_F32).log()
    S = s["scores"] = torch.softmax(logits, 1)
    member = torch.zeros((T, E), dtype=torch.bool, device="cuda")
    member.scatter_(1, torch.sort(S, dim=1, descending=True, stable=True).indices[:, :K], True)
    if M:
        f = member.sum(0)
        lo = f // M * M
        hi = (f + M - 1) // M * M
        keep = torch.where((hi - f < f - lo) & (hi <= T), hi, lo)
        order = torch.sort(torch.where(member, S + 2, S), dim=0, descending=True, stable=True).indices
        place = torch.empty_like(order)
        place.scatter_(0, order, torch.arange(T, device="cuda")[:, None].expand(T, E))
        member = place < keep[None, :]
    s["member"] = member
    return s


# ------------------------------------------------------------------ the plain form
def _scale_byte(amax):
    """amax = m 2^p, 1 <= m < 2: e = p - 8 for m <= 1.75, else p - 7, on the bits of the fp32 value."""
    bits = amax.to(_F32).contiguous().view(torch.int32)
    return (((bits + 0x1FFFFF) >> 23) - 8).clamp_min(1)


def _power(byte):
    return (byte << 23).contiguous().view(_F32)


def _quantize(x, block):
    """x fp32 [..., r, c] in blocks of block[0] x block[1]: e4m3 codes, and scale bytes (int32)."""
    r, c = x.shape[-2:]
    br, bc = block
    nr, nc = -(-r // br), -(-c // bc)
    p = torch.nn.functional.pad(x, (0, nc * bc - c, 0, nr * br - r)).unflatten(-2, (nr, br)).unflatten(-1, (nc, bc))
    byte = _scale_byte(p.abs().amax((-3, -1)))
    q = (p * _power(254 - byte)[..., :, None, :, None]).to(_E4M3)
    return q.flatten(-4, -3).flatten(-2, -1)[..., :r, :c], byte


def _dequantize(q, byte, block):
    r, c = q.shape[-2:]
    s = _power(byte).repeat_interleave(block[0], -2)[..., :r, :].repeat_interleave(block[1], -1)[..., :c]
    return q.to(_F32) * s


def _through(x, block):
    return _dequantize(*_quantize(x, block), block)


_ROW, _SQUARE = (1, 128), (128, 128)


def _halves(f, x, *a):
    """f on the gate and the up half of x's columns."""
    n = x.shape[-1] // 2
    return [f(x[..., :n], *a), f(x[..., n:], *a)]


def _plan(member, S):
    """The rows of every expert that has any, as tables padded to the longest: token of each slot (T: none) and its
    weight; and the slots of each token."""
    T = member.shape[0]
    w = S * member
    w = w / w.sum(1, keepdim=True).clamp_min(1e-30)
    experts = member.any(0).nonzero()[:, 0]
    m = member[:, experts].t()  # [hit, T]
    C = max(1, int(m.sum(1).max())) if m.numel() else 1
    tok = torch.sort(torch.where(m, torch.arange(T, device=m.device), T), dim=1).values[:, :C].contiguous()
    ws = torch.gather(torch.nn.functional.pad(w[:, experts].t(), (0, 1)), 1, tok)
    J = max(1, int(member.sum(1).max()))
    flat = tok.reshape(-1)
    live = (flat < T).nonzero()[:, 0]
    live = live[torch.sort(flat[live], stable=True).indices]
    t = flat[live]
    first = torch.cumsum(torch.bincount(t, minlength=T), 0) - torch.bincount(t, minlength=T)
    slots = torch.full((T, J), tok.numel(), dtype=torch.int64, device=m.device)
    slots[t, torch.arange(t.numel(), device=m.device) - first[t]] = live
    return {"experts": experts, "tok": tok, "w": ws, "slots": slots}


def _pad_row(x):
    return torch.nn.functional.pad(x, (0, 0, 0, 1))


def _per_token(rows, slots):
    """The sum over each token's rows [hit, C, cols]."""
    return _pad_row(rows.flatten(0, 1))[slots].sum(1)


def _forward(s, X, W1, W2, act):
    """X fp32; W1, W2 of the hit experts, fp32; act: what becomes of the activations before the second product."""
    p = s["plan"]
    H = torch.bmm(_pad_row(X)[p["tok"]], W1)
    if s["b1"] is not None:
        H += s["b1"][p["experts"]][:, None]
    n = H.shape[-1] // 2
    Y = torch.bmm(act(H[..., :n] * torch.sigmoid(H[..., :n]) * H[..., n:]), W2)
    if s["b2"] is not None:
        Y += s["b2"][p["experts"]][:, None]
    return H, _per_token(Y * p["w"][..., None], p["slots"])


def _backward(s, X, Hg, Hu, W1, W2):
    """Gradients from the kept values X and H = (Hg, Hu)."""
    p, T = s["plan"], s["T"]
    E, d, n2 = s["W1"].shape
    experts, tok, w = p["experts"], p["tok"], p["w"][..., None]
    sig = torch.sigmoid(Hg)
    A = Hg * sig * Hu
    dY = _pad_row(s["dO"].to(_F32))[tok]
    dAp = torch.bmm(dY, W2.transpose(1, 2).contiguous())
    dS = (dAp * A).sum(-1)
    if s["b2"] is not None:
        dS += (dY * s["b2"][experts][:, None]).sum(-1)
    dA = w * dAp
    dH = torch.cat([dA * Hu * sig * (1 + Hg * (1 - sig)), dA * Hg * sig], -1)
    rows = _pad_row(X)[tok]
    out = {"dW1": torch.zeros((E, d, n2), dtype=_BF16, device="cuda"),
           "dW2": torch.zeros((E, n2 // 2, d), dtype=_BF16, device="cuda")}
    out["dW1"][experts] = torch.bmm(rows.transpose(1, 2).contiguous(), dH).to(_BF16)
    out["dW2"][experts] = torch.bmm((w * A).transpose(1, 2).contiguous(), dY).to(_BF16)
    if s["b1"] is not None:
        out["db1"] = torch.zeros((E, n2), dtype=_BF16, device="cuda")
        out["db2"] = torch.zeros((E, d), dtype=_BF16, device="cuda")
        out["db1"][experts] = dH.sum(1).to(_BF16)
        out["db2"][experts] = (w * dY).sum(1).to(_BF16)
    # the router: dl = s (dS - sum s dS) over a token's experts
    live, ws = tok < T, p["w"]
    mean = torch.nn.functional.pad(_per_token((ws * dS)[..., None], p["slots"])[:, 0], (0, 1))
    dl = ws * (dS - mean[tok])
    dL = torch.zeros((T, E), dtype=_F32, device="cuda")
    dL[tok[live], experts[:, None].expand_as(tok)[live]] = dl[live]
    dX = _per_token(torch.bmm(dH, W1.transpose(1, 2).contiguous()), p["slots"]) + dL @ s["Wr"].to(_F32).t()
    out.update(dX=dX.to(_BF16), dWr=(X.t() @ dL).to(_BF16), dbias=dL.sum(0).to(_BF16))
    return out


def _run_plain(s):
    kind = s["kind"]
    if kind == "rows":
        q, byte = _quantize(s["X"].to(_F32), _ROW)
        return {"values": _dequantize(q, byte, _ROW).to(_BF16), "scale": byte.to(torch.uint8)}
    if kind == "experts":
        return {"W1": torch.cat(_halves(_through, s["W1"].to(_F32), _SQUARE), -1).to(_BF16),
                "W2": _through(s["W2"].to(_F32), _SQUARE).to(_BF16)}
    X, hit = s["X"].to(_F32), s["plan"]["experts"]
    if kind == "serve":
        W1 = torch.cat([_dequantize(q[hit], b[hit], _SQUARE) for q, b in s["q1"]], -1)
        W2 = _dequantize(s["q2"][0][hit], s["q2"][1][hit], _SQUARE)
        return {"O": _forward(s, _through(X, _ROW), W1, W2, lambda a: _through(a, _ROW))[1].to(_BF16)}
    W1, W2 = s["W1"][hit].to(_F32), s["W2"][hit].to(_F32)
    Xq = _through(X, _ROW) if kind == "quant" or s["keep_x"] else X
    if kind == "quant":
        H, O = _forward(s, Xq, torch.cat(_halves(_through, W1, _SQUARE), -1), _through(W2, _SQUARE),
                        lambda a: _through(a, _ROW))
    else:
        H, O = _forward(s, X, W1, W2, lambda a: a)
    Hg, Hu = _halves(_through, H, _ROW)
    return {"O": O.to(_BF16), **_backward(s, Xq if s["keep_x"] else X, Hg, Hu, W1, W2)}


# ------------------------------------------------------------------ states and passes
def prepare(case, seed):
    s = {**case, **_inputs(case, seed)}
    kind = case["kind"]
    member, S = s.pop("member", None), s.pop("scores", None)
    if own:
        from paper_2512_14080_amd import binding as B
        _prepare_own(B, s, case, S)
    elif kind not in ("rows", "experts"):
        s["plan"] = _plan(member, S)
        if kind == "serve":
            s["q1"] = _halves(lambda w: _quantize(w.to(_F32), _SQUARE), s["W1"])
            s["q2"] = _quantize(s["W2"].to(_F32), _SQUARE)
    if kind == "serve":  # the program holds the 8-bit weights only
        del s["W1"], s["W2"]
    return s


def _prepare_own(B, s, case, S):
    kind = case["kind"]

    def empty(*shape, dtype=_BF16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s["B"] = B
    if kind == "rows":
        rows, cols = case["rows"], case["cols"]
        s["q"], s["scale"] = empty(rows, cols, dtype=torch.uint8), empty(rows, B.scale_stride(cols), dtype=torch.uint8)
        s["values"] = empty(rows, cols)
        return
    T, K = case.get("T", 1), case.get("K", 1)
    d, n, E = case["d"], case["n"], case["E"]
    D = s["D"] = B.dims(T, d, n, E, K)
    if kind != "ckpt":
        s["qw"] = B.QExperts(D)
    if kind == "experts":
        s["out"] = {"W1": empty(E, d, 2 * n), "W2": empty(E, n, d)}
        return
    # the routing of these scores
    M = case["m_tile"]
    tc = B.Routing(D, T * K, B.MOE_ROUTING_SCORES_T if M else 0)
    tc.arrays()["scores"].copy_(S)
    B.moe_route(D, None, None, None, B.MOE_ROUTE_SCORES_IN | (B.MOE_ROUTE_WRITE_SCORES_T if M else 0), tc)
    s["r"] = tc
    if M:
        # an expert's own tokens in the selection's order: that of S + 2 in 32 bits, where scores less than 2^-22 apart are equal
        a = tc.arrays()
        picked = torch.zeros((T, E), dtype=torch.bool, device="cuda").scatter_(1, a["topk_idx"].long(), True)
        a["scores_t"].copy_(torch.where(picked, S + 2 - 2, S).t())
        s["r"] = B.Routing(D, B.moe_round_capacity(D, M))
        B.moe_round_tokens(D, M, "nearest", None, tc, s["r"])
    cap = s["r"].capacity
    s["O"] = empty(T, d)
    s["out"] = {"O": s["O"]}
    fwd = B.MOE_WS_FWD_CKPT if kind == "ckpt" else B.MOE_WS_FWD_QUANT
    s["ws_f"] = empty(B.moe_workspace_bytes(D, cap, fwd), dtype=torch.uint8)
    s["ckpt"] = db1 = db2 = None
    if kind == "serve":
        B.moe_quantize_experts(D, s["W1"], s["W2"], s["qw"])
    else:
        s["ckpt"] = B.Checkpoint(D, cap, keep_x=case["keep_x"])
        for k, t in (("dX", empty(T, d)), ("dW1", empty(E, d, 2 * n)), ("dW2", empty(E, n, d))):
            s[k] = s["out"][k] = t
        s["dWr"], s["dbias"] = empty(d, E, dtype=_F32), empty(E, dtype=_F32)
        if case["biases"]:
            db1 = s["db1"] = empty(E, 2 * n, dtype=_F32)
            db2 = s["db2"] = empty(E, d, dtype=_F32)
        s["ws_b"] = empty(B.moe_workspace_bytes(D, cap, B.MOE_WS_BWD_CKPT), dtype=torch.uint8)
    s["eb"] = B.expert_bias(s["b1"], s["b2"], db1, db2)


def _run_own(s):
    B, kind = s["B"], s["kind"]
    if kind == "rows":
        rows, cols = s["rows"], s["cols"]
        B.moe_quantize_rows(rows, cols, s["X"], s["q"], s["scale"])
        B.moe_dequantize_rows(rows, cols, s["q"], s["scale"], s["values"])
        return {"values": s["values"], "scale": s["scale"][:, :-(-cols // 128)]}
    D = s["D"]
    if kind == "experts":
        B.moe_quantize_experts(D, s["W1"], s["W2"], s["qw"])
        B.moe_dequantize_experts(D, s["qw"], s["out"]["W1"], s["out"]["W2"])
        return s["out"]
    if kind == "ckpt":
        B.moe_fwd_ckpt(D, s["X"], s["W1"], s["W2"], s["r"], s["ckpt"], s["O"], s["ws_f"], eb=s["eb"])
    else:
        if kind == "quant":
            B.moe_quantize_experts(D, s["W1"], s["W2"], s["qw"])
        B.moe_fwd_quant(D, s["X"], s["qw"], s["r"], s["ckpt"], s["O"], s["ws_f"], eb=s["eb"])
        if kind == "serve":
            return s["out"]
    B.moe_bwd_ckpt(D, s["dO"], None if s["keep_x"] else s["X"], s["ckpt"], s["W1"], s["W2"], s["Wr"], s["r"], s["dX"],
                   s["dW1"], s["dW2"], s["dWr"], s["dbias"], None, s["ws_b"], eb=s["eb"])
    # the small gradients go to 16 bits, as the program keeps the weights' own
    small = ("dWr", "dbias") + (("db1", "db2") if s["biases"] else ())
    return {**s["out"], **{k: s[k].to(_BF16) for k in small}}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def work(case):
    kind = case["kind"]
    if kind == "rows":
        # 16-bit values in, codes and scales out, and back
        v = case["rows"] * case["cols"]
        return {"bytes": 6 * v + 2 * v / 128, "flops": 3 * v}
    d, n, E = case["d"], case["n"], case["E"]
    if kind == "experts":
        v = 3 * E * d * n
        return {"bytes": 6 * v, "flops": 3 * v}
    T, K = case["T"], case["K"]
    P = T * K  # (rounding keeps the rows' number to within a few per cent)
    hit = E * (1 - (1 - K / E) ** T)  # experts that at least one token picks
    byts = 4 * T * d + 12 * P  # X, O; each row's token, weight and place
    flops = 6 * P * d * n
    if kind == "serve":
        return {"bytes": byts + 3 * hit * d * n, "flops": flops}  # codes of W1 and W2
    # 16-bit weights and W_r; dO; the kept H (and X); dX, dW1, dW2, dW_r
    byts += 6 * hit * d * n + 2 * d * E + 4 * T * d + 2 * P * n + case["keep_x"] * T * d + 6 * E * d * n + 2 * d * E
    if kind == "quant":
        byts += 3 * E * d * n  # the codes
    return {"bytes": byts, "flops": flops + 12 * P * d * n + 4 * T * d * E}


# ------------------------------------------------------------------ the definition in 64 bits
def _pow2(e):
    return ((e.long() + 1023) << 52).view(_F64)


def _round64(x, block):
    """x fp64 [r, c] through the 8-bit format, blocks of block[0] x block[1]."""
    r, c = x.shape
    amax = torch.nn.functional.max_pool2d(x.abs()[None, None], block, ceil_mode=True)[0, 0]
    m, p = torch.frexp(amax)  # m in [0.5, 1); 448 = 0.875 * 2^9
    e = (p - 8 - (m <= 0.875).int()).clamp_min(-126)
    e = torch.where(amax == 0, -126, e).repeat_interleave(block[0], 0)[:r].repeat_interleave(block[1], 1)[:, :c]
    v = x * _pow2(-e)
    step = _pow2(torch.frexp(v)[1].clamp_min(-5) - 4)  # three bits after the leading one, 2^-9 at the least
    return (v / step).round() * step * _pow2(e)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "rows":
        return {"values": _round64(s["X"].double(), (1, 128)), "scale": None}
    d, n, E = case["d"], case["n"], case["E"]
    square = (128, 128)

    def weights(e):
        w1, w2 = s["W1"][e].double(), s["W2"][e].double()
        return torch.cat([_round64(w1[:, :n], square), _round64(w1[:, n:], square)], 1), _round64(w2, square)

    if kind == "experts":
        w = [weights(e) for e in range(E)]
        return {"W1": torch.stack([a for a, _ in w]), "W2": torch.stack([b for _, b in w])}
    T, member = case["T"], s["member"]
    sw = s["scores"].double() * member
    sw = sw / sw.sum(1, keepdim=True).clamp_min(1e-300)
    X = s["X"].double()
    X8 = _round64(X, (1, 128))
    quant, train = kind != "ckpt", kind != "serve"
    Xf, Xb = X8 if quant else X, X8 if case["keep_x"] else X

    def zeros(*shape):
        return torch.zeros(shape, dtype=_F64, device="cuda")

    O, out = zeros(T, d), {}
    if train:
        dO, dX, dS = s["dO"].double(), zeros(T, d), zeros(T, E)
        out = {"dX": dX, "dW1": zeros(E, d, 2 * n), "dW2": zeros(E, n, d)}
        if case["biases"]:
            out.update(db1=zeros(E, 2 * n), db2=zeros(E, d))
    for e in range(E):
        t = member[:, e].nonzero()[:, 0]
        if not t.numel():
            continue
        w = sw[t, e][:, None]
        w1, w2 = s["W1"][e].double(), s["W2"][e].double()
        f1, f2 = weights(e) if quant else (w1, w2)
        h = Xf[t] @ f1
        if case["biases"]:
            h += s["b1"][e].double()
        a = h[:, :n] * torch.sigmoid(h[:, :n]) * h[:, n:]
        y = (_round64(a, (1, 128)) if quant else a) @ f2
        if case["biases"]:
            y += s["b2"][e].double()
        O.index_add_(0, t, w * y)
        if not train:
            continue
        gate, up = _round64(h[:, :n], (1, 128)), _round64(h[:, n:], (1, 128))
        sig = torch.sigmoid(gate)
        a, do = gate * sig * up, dO[t]
        da = do @ w2.t()
        dS[t, e] = (da * a).sum(1) + ((do * s["b2"][e].double()).sum(1) if case["biases"] else 0)
        da = w * da
        dh = torch.cat([da * up * sig * (1 + gate * (1 - sig)), da * gate * sig], 1)
        out["dW2"][e] = (w * a).t() @ do
        out["dW1"][e] = Xb[t].t() @ dh
        dX.index_add_(0, t, dh @ w1.t())
        if case["biases"]:
            out["db1"][e], out["db2"][e] = dh.sum(0), (w * do).sum(0)
    out["O"] = O
    if train:
        dL = sw * (dS - (sw * dS).sum(1, keepdim=True))
        dX += dL @ s["Wr"].double().t()
        out.update(dWr=Xb.t() @ dL, dbias=dL.sum(0))
    return out
