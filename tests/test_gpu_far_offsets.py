"""The dense products and moe_decode where byte offsets pass 31 and 32 bits: rows far apart, wide weights, long rows."""
import pytest

import dense_bounds as DB
from test_gpu_decode import Call, _inputs, _t
from test_gpu_linear import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,k,n,act,pad", [
    (5, 264, 136, "swiglu", 1 << 28),           # rows of 2.7 GB in all: past 31 bits
    (3, 72, 520, "gelu", (1 << 30) - 1024),     # the largest strides
    (130, 136, 72, "none", 1 << 25),            # 8.7 GB, several tiles
    (4, 40960, 32768, "silu", 0),               # a W of 2.7 GB, few rows
    (40, 16384, 40960, "swiglu", 0),            # of 2.7 GB, gate and up columns
])
def test_linear(T, k, n, act, pad):
    torch = _t()
    c = Case(T, k, n, act, pad)
    c.fwd()
    c.bwd()
    c.guards()
    print("shares of the bounds:", c.check_fwd(), c.check_bwd(), flush=True)
    del c
    torch.cuda.empty_cache()


DECODE = [
    (2, 262144, 64, 8, 2),     # the longest sums over d, most column tiles
    (20, 131072, 64, 8, 2),
    (3, 8192, 65472, 8, 2),    # an expert's W1 within 2 MB of 2^31 bytes
    (40, 8192, 32768, 8, 2),
]


@pytest.mark.parametrize("T,d,n,E,K", DECODE)
def test_decode(T, d, n, E, K):
    """By element, whose bounds are wide for sums so long, and by token in the norm: O's rounding is at most 2^-8 of it, and
    A's, 2^-8 of its values and independent of each other, add as their squares to about as much of Y."""
    torch = _t()
    X, Wr, bias, W1, W2, b1, b2, R = _inputs(T, d, n, E, K, 100 + T + d)
    W1.mul_(d ** -0.5 / 0.05)
    W2.mul_(n ** -0.5 / 0.05)
    idx, w, ew, gap = DB.select(X, Wr, bias, K)
    ref, bound = DB.decode(X, W1, W2, b1, b2, R, idx, w, ew)
    call = Call(T, d, n, E, K)
    call(X, Wr, bias, W1, W2, b1, b2, R)
    O, gi, gw = call.results()
    assert gap > 2 ** -12 and torch.equal(gi.long(), idx)
    DB.within(gw, w, ew, "weights")
    off = (O.double() - ref).norm(dim=1) / ref.norm(dim=1)
    print("share of the bound:", DB.within(O, ref, bound, "O"), "off by", off.max().item(), flush=True)
    assert off.max() <= 2 * 2.0 ** -8
    del X, Wr, W1, W2, ref, bound, call
    torch.cuda.empty_cache()


def _through(x, block):
    """x in 64 bits through the 8-bit block format: the least power of two that holds a block's values up to 448 times it, and
    four significant bits of each, to nearest even, down to 2^-9."""
    torch = _t()

    def pow2(e):  # (exactly, whatever the device's pow is off by)
        return ((e.long() + 1023) << 52).view(torch.float64)

    r, c = x.shape
    m, p = torch.frexp(torch.nn.functional.max_pool2d(x.abs()[None, None], block, ceil_mode=True)[0, 0])  # 448 = 0.875 2^9
    e = (p - 8 - (m <= 0.875).int()).clamp_min(-126).repeat_interleave(block[0], 0)[:r].repeat_interleave(block[1], 1)[:, :c]
    v = x * pow2(-e)
    step = pow2(torch.frexp(v)[1].clamp_min(-5) - 4)
    return (v / step).round() * step * pow2(e)


@pytest.mark.parametrize("T,d,n,E,K", DECODE)
def test_decode_quant(T, d, n, E, K):
    """By token in the norm: O's rounding is at most 2^-8 of it.  Sums of d products in fp32 are some d^0.5 2^-24 off, 3e-5 for
    the longest; of A's codes, steps of up to 2^-3 apart and 2^-4 at the least, as many as 1e-3 are then on the other side,
    in the norm 2^-4 (1e-3)^0.5 = 2e-3."""
    torch = _t()
    X, Wr, bias, W1, W2, b1, b2, _ = _inputs(T, d, n, E, K, 100 + T + d, residual=False)
    W1.mul_(d ** -0.5 / 0.05)
    W2.mul_(n ** -0.5 / 0.05)
    call = Call(T, d, n, E, K, quant=True)
    B = call.B
    q = B.QExperts(call.D)
    B.moe_quantize_experts(call.D, W1, W2, q)
    call(X, Wr, bias, W1, W2, b1, b2, None, q=q)
    O, gi, _ = call.results()
    idx, w, _, gap = DB.select(X, Wr, bias, K)
    assert gap > 2 ** -12 and torch.equal(gi.long(), idx)
    x8, sq = _through(X.double(), (1, 128)), (128, 128)
    ref = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    for e in torch.unique(idx).tolist():
        t, j = (idx == e).nonzero(as_tuple=True)
        h = [x8[t] @ _through(W1[e][:, half].double(), sq) for half in (slice(0, n), slice(n, 2 * n))]
        a = _through(torch.nn.functional.silu(h[0]) * h[1], (1, 128))
        ref.index_add_(0, t, w[t, j][:, None] * (a @ _through(W2[e].double(), sq)))
    off = (O.double() - ref).norm(dim=1) / ref.norm(dim=1)
    print("off by", off.max().item(), flush=True)
    assert off.max() <= 2.0 ** -8 + 2e-3
    del X, Wr, W1, W2, q, call
    torch.cuda.empty_cache()
