"""layer.SharedExpert on rows that are further apart than they are long: the results of contiguous rows, bit for bit, and
nothing beside the rows."""
import pytest

pytestmark = pytest.mark.gpu


def _t():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _apart(t, pad, fill):
    """t's values in rows that are `pad` further apart, with `fill` between them: (buffer, view)."""
    torch = _t()
    rows, cols = t.shape
    buf = torch.full((rows, cols + pad), fill, dtype=t.dtype, device="cuda")
    buf[:, :cols] = t
    return buf, buf[:, :cols]


@pytest.mark.parametrize("T,d,m", [(1, 256, 200), (5, 512, 264), (40, 1000, 136), (300, 256, 520)])
def test_rows_apart(T, d, m):
    """Each operand with a stride of its own (X, dX and G with one); R and G in place too.  The sums are the same ones in
    the same order, so the results are equal."""
    torch = _t()
    from paper_2512_14080_amd.layer import SharedExpert
    g = torch.Generator(device="cuda").manual_seed(T + d)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    Wu, Wd = normal(d, 2 * m, std=d ** -0.5), normal(m, d, std=m ** -0.5)
    bu, bd = (torch.randn(s, generator=g, device="cuda") * 0.1 for s in (2 * m, d))
    X, R, dY, G = (normal(T, d) for _ in range(4))
    s = SharedExpert(T, Wu, Wd, bu, bd, train=True)
    grads = ("dWu", "dWd", "dbu", "dbd")
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    s.forward(X, Y, R)
    s.backward(dY, X, dX, G)
    torch.cuda.synchronize()
    want = {n: getattr(s, n).clone() for n in grads}
    nan = float("nan")
    _, x = _apart(X, 8, nan)
    _, r = _apart(R, 24, nan)
    _, dy = _apart(dY, 16, nan)
    _, gg = _apart(G, 8, nan)
    ybuf, y = _apart(torch.zeros_like(Y), 40, 7.0)
    xbuf, dx = _apart(torch.zeros_like(dX), 8, 7.0)
    s.forward(x, y, r)
    s.backward(dy, x, dx, gg)
    torch.cuda.synchronize()
    assert torch.equal(y, Y) and torch.equal(dx, dX)
    assert all(torch.equal(getattr(s, n), want[n]) for n in grads)
    assert bool((ybuf[:, d:] == 7.0).all()) and bool((xbuf[:, d:] == 7.0).all())
    # in place
    s.forward(x, r, r)
    s.backward(dy, x, gg, gg)
    torch.cuda.synchronize()
    assert torch.equal(r, Y) and torch.equal(gg, dX)


def test_decode_of_a_layer_too_long():
    """More tokens than the call takes: the library's error, with nothing launched."""
    torch = _t()
    from paper_2512_14080_amd import binding as B
    from paper_2512_14080_amd import workloads as W
    from paper_2512_14080_amd.layer import DeviceLayer
    cfg = W.MoEConfig("decode", T=65, d=128, n=64, E=8, K=2, m_tile=64)
    layer = DeviceLayer(W.make_inputs(cfg, 3))
    layer.O.fill_(7.0)
    with pytest.raises(B.MoEError, match="at most 64"):
        layer.decode()
    torch.cuda.synchronize()
    assert bool((layer.O == 7.0).all())
