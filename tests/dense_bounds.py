"""Definitions in 64 bits of moe_decode and the dense products, each with a bound of the kernels' error by element.

The bounds count, for every value, what the kernels round: a rounding to bf16 is off by at most U = 2^-8 of the value,
a sum of n products in fp32 by n 2^-24 of the sum of their magnitudes (any order), and exp, the reciprocal and erf by
F = 2^-20 of their results (a few units in the last place, with the arithmetic around them)."""
import torch

U, F = 2.0 ** -8, 2.0 ** -20


def E(n):
    return (n + 8) * 2.0 ** -24


def act(h, name):
    """act(h), its largest slope on either side (for an error of h) and its derivative."""
    if name == "none":
        return h, torch.ones_like(h), torch.ones_like(h)
    if name == "relu":
        return torch.relu(h), torch.ones_like(h), (h > 0).double()
    if name == "silu":
        s = torch.sigmoid(h)
        return h * s, torch.full_like(h, 1.1), s * (1 + h * (1 - s))
    if name == "gelu":
        c = 0.5 * (1 + torch.erf(h / 2 ** 0.5))
        return h * c, torch.full_like(h, 1.13), c + h * torch.exp(-h * h / 2) / (2 * torch.pi) ** 0.5
    raise ValueError(name)


def linear(X, W, b, R, name):
    """(H, bound of H, Y, bound of Y); H's before its rounding."""
    X, W = X.double(), W.double()
    k = X.shape[1]
    H, m = X @ W, X.abs() @ W.abs()
    if b is not None:
        H, m = H + b.double(), m + b.double().abs()
    e = E(k) * m
    if name == "swiglu":
        n = W.shape[1] // 2
        g, u = H[:, :n], H[:, n:]
        s, _, _ = act(g, "silu")
        Y = s * u
        eY = 1.1 * e[:, :n] * (u.abs() + e[:, n:]) + s.abs() * e[:, n:] + F * Y.abs()
    else:
        Y, slope, _ = act(H, name)
        eY = slope * e + F * (Y.abs() + H.abs())
    if R is not None:
        Y = Y + R.double()
        eY = eY + 2.0 ** -23 * Y.abs()
    return H, e + U * (H.abs() + e), Y, eY + U * (Y.abs() + eY)


def linear_grad(dY, X, W, H, G, name):
    """{dX, dW, db: (value, bound)} at the kept H (None: no activation)."""
    dY, X, W = dY.double(), X.double(), W.double()
    if name == "none":
        dP, e, r = dY, torch.zeros_like(dY), 0.0
    elif name == "swiglu":
        n = H.shape[1] // 2
        g, u = H[:, :n].double(), H[:, n:].double()
        s = torch.sigmoid(g)
        dP = torch.cat([dY * u * s * (1 + g * (1 - s)), dY * g * s], 1)
        e = F * torch.cat([dY * u * s * (1 + g.abs()), dY * g * s], 1).abs()
        r = U
    else:
        h = H.double()
        dP = dY * act(h, name)[2]
        e = F * dY.abs() * (1 + h.abs())
        r = U
    N, T = dP.shape[1], dP.shape[0]
    q = e + r * (dP.abs() + e)  # of dP as the products read it
    dX, m = dP @ W.t(), dP.abs() @ W.abs().t()
    eX = q @ W.abs().t() + E(N) * (m + q @ W.abs().t())
    if G is not None:
        dX = dX + G.double()
        eX = eX + 2.0 ** -23 * dX.abs()
    dW, mW, qW = X.t() @ dP, X.abs().t() @ dP.abs(), X.abs().t() @ q
    eW = qW + E(T) * (mW + qW)
    db, eb = dP.sum(0), e.sum(0) + E(T) * (dP.abs().sum(0) + e.sum(0))
    return {"dX": (dX, eX + U * (dX.abs() + eX)), "dW": (dW, eW + U * (dW.abs() + eW)), "db": (db, eb)}


def select(X, Wr, bias, K):
    """(experts, weights, bound of the weights, the least distance of two neighbours among the K + 1 best logits)."""
    X, Wr = X.double(), Wr.double()
    l = X @ Wr
    m = X.abs() @ Wr.abs()
    if bias is not None:
        l, m = l + bias.double(), m + bias.double().abs().nan_to_num(posinf=0.0)
    v, idx = torch.sort(l, dim=1, descending=True, stable=True)
    gap = (v[:, :K] - v[:, 1:K + 1]).min().item() if K < l.shape[1] else float("inf")
    w = torch.softmax(v[:, :K], 1)
    # an error d of a logit moves a weight by at most 2 d of it
    ew = w * (2 * E(X.shape[1]) * m.amax(1, keepdim=True) + F)
    return idx[:, :K], w, ew, gap


def decode(X, W1, W2, b1, b2, R, idx, w, ew):
    """(O, its bound) for the given selection."""
    T, d = X.shape
    n = W2.shape[1]
    O, e = torch.zeros((T, d), dtype=torch.float64, device=X.device), None
    e = torch.zeros_like(O)
    x = X.double()
    for ex in torch.unique(idx).tolist():
        t, j = (idx == ex).nonzero(as_tuple=True)
        _, _, a, ea = linear(x[t], W1[ex], None if b1 is None else b1[ex], None, "swiglu")  # (ea: with A's rounding)
        w2 = W2[ex].double()
        y, m = a @ w2, a.abs() @ w2.abs()
        if b2 is not None:
            y, m = y + b2[ex].double(), m + b2[ex].double().abs()
        ey = ea @ w2.abs() * (1 + E(n)) + E(n) * m
        s, es = w[t, j][:, None], ew[t, j][:, None]
        O.index_add_(0, t, s * y)
        e.index_add_(0, t, s * ey + es * (y.abs() + ey) + 2.0 ** -20 * s * y.abs())
    if R is not None:
        O = O + R.double()
    e = e + 2.0 ** -20 * O.abs()
    return O, e + U * (O.abs() + e)


def within(got, ref, bound, what=""):
    """Asserts |got - ref| <= bound by element; returns the largest share of the bound that is used."""
    d = (got.double() - ref).abs()
    ok = d <= bound
    assert bool(ok.all()), f"{what}: {int((~ok).sum())} of {ok.numel()} past the bound, worst {(d / bound).max().item():.3g}"
    return (d / bound.clamp_min(1e-300)).max().item()
