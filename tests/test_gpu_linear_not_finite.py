"""The dense product's gradients where values are not finite."""
import pytest

from test_gpu_linear import Case, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("T", [5, 40, 300])
def test_relu_stops_what_is_not_finite(T, value):
    """dY that is not finite at units that are off (H <= 0) leaves no trace: the gradients are those of 0 there."""
    torch = _t()
    c = Case(T, 264, 136, "relu", 8)
    c.fwd()
    torch.cuda.synchronize()
    off = c.H <= 0
    assert bool(off.any(1).all()) and not bool(off.all(1).any())  # (every row has units of both kinds)
    c.dY[off] = value
    c.bwd()
    c.guards()
    got = [t.clone() for t in (c.dX, c.dW, c.db)]
    c.dY[off] = 0
    c.bwd()
    c.guards()
    assert all(torch.equal(a, b) for a, b in zip(got, (c.dX, c.dW, c.db)))
    c.check_bwd()


def test_relu_lets_through_what_is_not_finite():
    """At a unit that is on it reaches its row of dX, its column of dW and of db, and no others."""
    torch = _t()
    c = Case(40, 264, 136, "relu", 8)
    c.fwd()
    torch.cuda.synchronize()
    t, n = (int(i) for i in (c.H > 0).nonzero()[70])
    c.dY[t, n] = float("inf")
    c.bwd()
    c.guards()
    rows, cols = torch.arange(40) != t, torch.arange(136) != n
    assert not bool(torch.isfinite(c.dX[t]).any()) and bool(torch.isfinite(c.dX[rows]).all())
    assert not bool(torch.isfinite(c.dW[:, n]).any()) and bool(torch.isfinite(c.dW[:, cols]).all())
    assert c.db[n] == float("inf") and bool(torch.isfinite(c.db[:136][cols]).all())
