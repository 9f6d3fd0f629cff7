"""The dense products on the GPU against their definition in 64 bits (dense_bounds), by element."""
import pytest

import dense_bounds as DB

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu", "swiglu"]


def _t():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


class Case:
    """Inputs and outputs of one product; what lies between the rows is NaN (inputs) or a mark (outputs)."""

    def __init__(self, T, k, n, act, pad=0, bias=True, residual=True, seed=0):
        torch = _t()
        from paper_2512_14080_amd import binding as B
        self.B, self.T, self.k, self.n, self.act, self.pad = B, T, k, n, act, pad
        self.N = N = 2 * n if act == "swiglu" else n
        self.L = B.linear_dims(T, k, n, act, *((k + pad, n + pad, n + pad) if pad else (0, 0, 0)))
        g = torch.Generator(device="cuda").manual_seed(seed + T + 7 * k + 13 * n)

        def rows(cols, std=1.0, fill=float("nan")):
            buf = torch.full((T * (cols + pad) + 64,), fill, dtype=torch.bfloat16, device="cuda")
            v = buf[:T * (cols + pad)].view(T, cols + pad)[:, :cols]
            if std:
                v.copy_(torch.randn((T, cols), generator=g, device="cuda") * std)
            return buf, v

        self._x, self.X = rows(k)
        self._r, self.R = rows(n) if residual else (None, None)
        self._dy, self.dY = rows(n)
        self._g, self.G = rows(k) if residual else (None, None)
        self._y, self.Y = rows(n, 0, 7.0)
        self._dx, self.dX = rows(k, 0, 7.0)
        w = torch.full((k * N + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
        self._w, self.W = w, w[:k * N].view(k, N)
        self.W.copy_(torch.randn((k, N), generator=g, device="cuda") * k ** -0.5)
        self.b = torch.randn((N,), generator=g, device="cuda") * 0.5 if bias else None
        self._h = torch.full((T * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        self.H = self._h[:T * N].view(T, N)
        self._dw = torch.full((k * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        self.dW = self._dw[:k * N].view(k, N)
        self.db = torch.full((N + 16,), 7.0, device="cuda")
        need = [B.moe_linear_workspace_bytes(self.L, i) for i in (B.MOE_WS_LINEAR_FWD, B.MOE_WS_LINEAR_BWD)]
        self.buf = [torch.full((m + 512,), 0x7F, dtype=torch.uint8, device="cuda") for m in need]
        self.off = [(-b.data_ptr()) % 256 for b in self.buf]
        self.need = need
        self.ws = [b[o:o + m] for b, o, m in zip(self.buf, self.off, need)]

    def fwd(self, keep=True, stream=None, R="own", Y=None):
        self.B.moe_linear_fwd(self.L, self._x, self._w, self.b, self._r if R == "own" else R, self.H if keep else None,
                              self._y if Y is None else Y, self.ws[0], stream)

    def bwd(self, dX=True, dW=True, db=True, stream=None):
        self.B.moe_linear_bwd(self.L, self._dy, self._x, self._w, None if self.act == "none" else self.H, self._g,
                              self._dx if dX else None, self.dW if dW else None, self.db if db else None, self.ws[1],
                              stream)

    def guards(self):
        torch = _t()
        torch.cuda.synchronize()
        for buf, v, cols in ((self._y, self.Y, self.n), (self._dx, self.dX, self.k)):
            assert bool((buf[self.T * (cols + self.pad):] == 7.0).all())
            if self.pad:
                assert bool((buf[:self.T * (cols + self.pad)].view(self.T, -1)[:, cols:] == 7.0).all())
        assert bool((self._h[self.T * self.N:] == 7.0).all()) and bool((self._dw[self.k * self.N:] == 7.0).all())
        assert bool((self.db[self.N:] == 7.0).all())
        for b, o, m in zip(self.buf, self.off, self.need):
            assert bool((b[o + m:] == 0x7F).all())

    def check_fwd(self):
        H, eH, Y, eY = DB.linear(self.X, self.W, self.b, self.R, self.act)
        use = DB.within(self.Y, Y, eY, "Y")
        DB.within(self.H, H, eH, "H")
        return use

    def check_bwd(self, dX=True, dW=True, db=True):
        ref = DB.linear_grad(self.dY, self.X, self.W, None if self.act == "none" else self.H, self.G, self.act)
        use = {}
        for name, on, got in (("dX", dX, self.dX), ("dW", dW, self.dW), ("db", db, self.db[:self.N])):
            if on:
                use[name] = DB.within(got, *ref[name], name)
        return use


# rows: streamed up to 64 (in tiles of 4, 8 and 16 rows), tiled beyond; sizes that end inside every kind of tile
SIZES = [(1, 8, 8, 0), (1, 1024, 1536, 0), (1, 4096, 264, 8), (2, 1000, 8, 0), (4, 136, 2048, 16), (5, 264, 520, 8), (8, 72, 1032, 0),
         (9, 904, 136, 8), (16, 256, 256, 0), (17, 328, 264, 24), (31, 64, 200, 0), (33, 1000, 392, 8), (64, 512, 1024, 0),
         (65, 64, 64, 0), (100, 4096, 128, 8), (129, 136, 264, 0), (255, 256, 256, 0), (256, 72, 512, 8), (257, 520, 520, 0),
         (700, 200, 1032, 8), (1024, 1024, 768, 0), (3001, 8, 8, 0), (2500, 264, 40, 8)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,k,n,pad", SIZES)
def test_linear(T, k, n, pad, act):
    c = Case(T, k, n, act, pad, bias=(T + k) % 3 != 0, residual=(T + n) % 4 != 0)
    c.fwd()
    c.bwd(db=True)
    c.guards()
    print("shares of the bounds:", c.check_fwd(), c.check_bwd(), flush=True)
    first = [t.clone() for t in (c.Y, c.H, c.dX, c.dW, c.db)]
    c.fwd()
    c.bwd()
    c.guards()
    torch = _t()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.Y, c.H, c.dX, c.dW, c.db)))


@pytest.mark.parametrize("T,k,n,act", [(20000, 512, 256, "swiglu"), (4100, 1544, 2056, "gelu"), (70, 8192, 512, "silu"),
                                       (48, 8192, 2048, "none"), (9000, 256, 64, "relu"), (3, 16384, 1024, "swiglu"),
                                       (1777, 72, 14336, "swiglu"), (1777, 28672, 72, "relu")])
def test_large(T, k, n, act):
    """Many tiles and rounds, sliced reductions, split gradients, whole rounds of columns apart (the last two)."""
    c = Case(T, k, n, act, 8)
    c.fwd()
    c.bwd()
    c.guards()
    print("shares of the bounds:", c.check_fwd(), c.check_bwd(), flush=True)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,k,n", [(17, 520, 136), (33, 264, 264), (100, 1032, 520), (257, 512, 512), (500, 2056, 72),
                                   (1024, 64, 64), (130, 72, 4104), (2049, 72, 40)])
def test_row_groups(T, k, n, act):
    """Streamed products whose rows go to several groups, the last one short, with and without slices of k."""
    c = Case(T, k, n, act, 8, bias=T % 2 == 0, residual=T % 3 != 0)
    c.fwd()
    c.bwd()
    c.guards()
    print("shares of the bounds:", c.check_fwd(), c.check_bwd(), flush=True)


@pytest.mark.parametrize("T", [3, 50, 300])
def test_parts(T):
    """Each output alone, without H, without bias and residual, R in place, on another stream."""
    torch = _t()
    for act in ACTS:
        c = Case(T, 264, 136, act, 8)
        c.fwd()
        c.bwd()
        c.guards()
        Y, ref = c._y.clone(), {k: getattr(c, k).clone() for k in ("dX", "dW", "db")}
        c._y.fill_(7.0)
        c.fwd(keep=False)
        c.guards()
        assert torch.equal(c._y, Y)
        for name in ref:
            getattr(c, "_dx" if name == "dX" else name).fill_(7.0)
            c.bwd(**{k: k == name for k in ref})
            c.guards()
            assert torch.equal(getattr(c, name), ref[name]), (act, name)
        side = torch.cuda.Stream()
        out = c._r.clone()
        side.wait_stream(torch.cuda.current_stream())
        c.fwd(R=out, Y=out, stream=side)
        side.synchronize()
        n = T * (136 + 8)
        assert torch.equal(out[:n].view(T, -1)[:, :136], Y[:n].view(T, -1)[:, :136])
        c = Case(T, 264, 136, act, 0, bias=False, residual=False)
        c.fwd()
        c.bwd()
        c.check_fwd()
        c.check_bwd()


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    """<dX, v> + <dW, M> + <db, q> and the difference of <dY, Y> in 64 bits along (v, M, q): the central difference is off by
    h^2 / 6 of the third derivative (h = 1e-4: below 1e-6 here), the kernel's side by its bounds."""
    torch = _t()
    c = Case(40, 72, 56, act, 0, residual=False, seed=3)
    if act == "relu":  # (away from the corner, where there is no derivative)
        c.b.add_(torch.where(torch.rand(c.N, device="cuda") < 0.5, -6.0, 6.0))
    c.fwd()
    # the kept H is rounded: the derivative is taken there, of the activation; so the products' part from H itself
    c.bwd()
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(1)
    v, M, q = (torch.randn(s, generator=g, device="cuda", dtype=torch.float64) for s in ((40, 72), (72, c.N), (c.N,)))
    X, W, b, dY = c.X.double(), c.W.double(), c.b.double(), c.dY.double()

    def loss(h):
        # H at the kept values, moved along the direction
        d = (X + h * v) @ (W + h * M) - X @ W + h * q
        H = (c.H.double() if act != "none" else X @ W + b) + d
        if act == "swiglu":
            n = c.n
            return (dY * torch.nn.functional.silu(H[:, :n]) * H[:, n:]).sum()
        return (dY * DB.act(H, act)[0]).sum()

    h = 1e-4
    diff = ((loss(h) - loss(-h)) / (2 * h)).item()
    ref = DB.linear_grad(c.dY, c.X, c.W, None if act == "none" else c.H, None, act)
    along = ((c.dX.double() * v).sum() + (c.dW.double() * M).sum() + (c.db[:c.N].double() * q).sum()).item()
    tol = ((ref["dX"][1] * v.abs()).sum() + (ref["dW"][1] * M.abs()).sum() + (ref["db"][1] * q.abs()).sum()).item()
    size = ((ref["dX"][0] * v).abs().sum() + (ref["dW"][0] * M).abs().sum()).item()
    print(act, diff, along, tol, flush=True)
    assert abs(diff - along) <= tol + 1e-6 * size


def test_not_finite():
    """A row of X that is not finite stays in its row of Y; Inf beside the last columns of W never enters."""
    torch = _t()
    for T, k, n in ((6, 264, 136), (40, 1000, 72), (300, 328, 200)):
        c = Case(T, k, n, "silu", 8)
        c.fwd()
        torch.cuda.synchronize()
        Y = c.Y.clone()
        c.X[2, 3] = float("inf")
        c.fwd()
        torch.cuda.synchronize()
        rest = torch.arange(T) != 2
        assert torch.equal(c.Y[rest], Y[rest]) and not bool(torch.isfinite(c.Y[2]).all())
        c.X[2, 3] = float("nan")
        c.fwd()
        torch.cuda.synchronize()
        assert torch.equal(c.Y[rest], Y[rest]) and bool(torch.isnan(c.Y[2]).all())


@pytest.mark.parametrize("T", [2, 90])
def test_step_in_a_graph(T):
    """A captured step replayed between eager ones (of other sizes, on the same workspace) with changing inputs."""
    torch = _t()
    c, other = Case(T, 512, 264, "swiglu", 0), Case(T + 1, 264, 512, "gelu", 0)
    if c.need[1] > other.need[1]:
        other.ws[1] = c.ws[1]
    for x in (c, other):
        x.fwd()
        x.bwd()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.fwd()
        c.bwd()
    for rep in range(4):
        c.X.copy_(torch.randn((T, 512), device="cuda"))
        c.dY.copy_(torch.randn((T, 264), device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (c.Y, c.H, c.dX, c.dW, c.db)]
        other.fwd()
        other.bwd()
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (c.Y, c.H, c.dX, c.dW, c.db))), rep
