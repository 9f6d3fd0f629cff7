"""The codes in which moe_decode_quant holds A, each one: its up-projection sums in fp32, and where such sums are exact the
codes are the definition's.

X and W1 are integers of four significant bits up to 256, which the block format holds exactly, and the magnitudes of any
sum of their products stay below 2^24: H is the same integer in fp32, whatever the order.  The gate is 128 or 1024, where
SiLU is the identity, so A is 128 or 1024 times H's up column; and these lie one step of the integers (2^-18 of the value
and less) from a border of the codes, above or below it, or at the border of a block's scale.  A sum with fewer bits puts
some of them on the other side, which is 1/15 of the value or more.

W2 hands every expert's A to columns of their own, so an element of O is a weight times one of A's values: rounded once, to
2^-8, behind fp32 products (2^-20) and the weight's own error."""
import pytest

import dense_bounds as DB
from oracle import block8
from test_gpu_decode import Call, _t

pytestmark = pytest.mark.gpu

TUNE, GATE = 10, 10  # rows of W1 that place H's columns; the row that forms the gate


def _placed(delta):
    """[TUNE, n] weights w with sum over r of xt[r] w[r] = delta, as far as they reach, and xt."""
    torch = _t()
    xt = torch.tensor([256.0] * 7 + [256.0, 16.0, 1.0], dtype=torch.float64, device="cuda")
    w = torch.zeros((TUNE, delta.numel()), dtype=torch.float64, device="cuda")
    left = delta.clone()
    for r in range(6):
        w[r] = 240 * (left / 61440).round().clamp(-1, 1)
        left -= 256 * w[r]
    w[6] = 16 * (left / 4096).round().clamp(-8, 8)
    left -= 256 * w[6]
    for r, x in ((7, 256.0), (8, 16.0), (9, 1.0)):
        w[r] = (left / x).round().clamp(-8, 8)
        left -= x * w[r]
    return w, xt, left == 0


def _integers(g, shape):
    """m 2^p with m from 1 to 15 and p from 0 to 4, either sign."""
    torch = _t()
    m = torch.randint(1, 16, shape, generator=g, device="cuda").double()
    p = torch.randint(0, 5, shape, generator=g, device="cuda").double()
    s = torch.randint(0, 2, shape, generator=g, device="cuda").double() * 2 - 1
    return s * m * 2 ** p


@pytest.mark.parametrize("T,d,n,E,K", [
    (1, 1536, 256, 128, 8),   # by token, k in slices
    (1, 1024, 128, 8, 8),
    (6, 1536, 256, 128, 8),   # by group from here on, narrow tiles
    (7, 512, 1088, 16, 4),    # blocks of k that end early
    (12, 1024, 128, 8, 8),
    (20, 1536, 192, 16, 4),
    (24, 1024, 64, 64, 16),
    (40, 1024, 128, 8, 8),    # two row blocks, two passes
    (64, 1536, 256, 128, 8),
])
def test_codes_of_a(T, d, n, E, K):
    torch = _t()
    from paper_2512_14080_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(T + d + n)
    bf16, f64 = torch.bfloat16, torch.float64
    X = _integers(g, (3 * T + 16, d))
    X[:, :TUNE] = _placed(torch.zeros(1, dtype=f64, device="cuda"))[1]
    X[:, GATE] = 128
    Wr = (torch.randn((d, E), generator=g, device="cuda") * (0.02 * d ** -0.5)).to(bf16)
    best = torch.sort(X @ Wr.double(), dim=1, descending=True).values[:, :K + 1]
    X = X[(best[:, :-1] - best[:, 1:]).amin(1) > 2 ** -9][:T].contiguous()
    assert X.shape[0] == T
    idx, w, ew, gap = DB.select(X.to(bf16), Wr, None, K)
    cols = min(d // E, n)  # of an expert
    W1, W2 = torch.zeros((E, d, 2 * n), dtype=bf16, device="cuda"), torch.zeros((E, n, d), dtype=bf16, device="cuda")
    ref, bound = torch.zeros((T, d), dtype=f64, device="cuda"), torch.zeros((T, d), dtype=f64, device="cuda")
    near = total = 0
    for e in torch.unique(idx).tolist():
        t, j = (idx == e).nonzero(as_tuple=True)
        up = _integers(g, (d, n))
        up[:TUNE + 1] = 0
        h = X[t[0]] @ up  # of the expert's first token, whose columns are placed
        size = 2 ** torch.floor(torch.log2(h.abs().clamp_min(1)))
        aim = (torch.floor(8 * h.abs() / size) + 0.5) * size / 8  # between two codes
        scale = torch.arange(n, device="cuda") % 128 == 0
        aim = torch.where(scale, 1.75 * size, aim)  # the largest that the block's scale holds
        side = torch.randint(0, 2, (n,), generator=g, device="cuda").double()
        aim = aim + torch.where(scale, side, 2 * side - 1)
        up[:TUNE], _, done = _placed(torch.sign(h) * aim - h)
        up[:, ~done & scale] *= 0
        gate = torch.where(scale, 8.0, 1.0).double()
        W1[e, :, n:] = up.to(bf16)
        W1[e, GATE, :n] = gate.to(bf16)
        assert torch.equal(W1[e, :, n:].double(), up) and ((X[t].abs() @ up.abs()).max().item() < 2 ** 24)
        a = (128 * gate) * (X[t] @ up)
        w1 = torch.from_numpy(block8.through(up.cpu().numpy(), (128, 128))).cuda()
        assert torch.equal(w1, up)  # (held exactly)
        a8 = torch.from_numpy(block8.through(a.cpu().numpy())).cuda()
        take = torch.randperm(n, generator=g, device="cuda")[:cols]
        take[0] = 0
        if take[1:].eq(0).any():
            take[1:][take[1:] == 0] = (set(range(n)) - set(take.tolist())).pop()
        out = e * cols + torch.arange(cols, device="cuda")
        W2[e, take, out] = 1.0
        y = w[t, j][:, None] * a8[:, take]
        ref[t[:, None], out] = y
        bound[t[:, None], out] = DB.U * y.abs() + 2.0 ** -20 * y.abs() + ew[t, j][:, None] * 1.01 * a8[:, take].abs()
        near += int(done[take].sum())
        total += cols
    assert torch.equal(torch.from_numpy(block8.through(X.cpu().numpy())).cuda(), X)
    assert near >= 0.9 * total, (near, total)
    call = Call(T, d, n, E, K, quant=True)
    q = B.QExperts(call.D)
    B.moe_quantize_experts(call.D, W1, W2, q)
    call(X.to(bf16).contiguous(), Wr, None, W1, W2, None, None, None, q=q)
    O, gi, _ = call.results()
    assert gap > 2 ** -10 and torch.equal(gi.long(), idx)
    print("placed", near, "of", total, flush=True)
    DB.within(O, ref, bound, "O")
