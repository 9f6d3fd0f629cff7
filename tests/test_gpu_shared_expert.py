"""The routed experts and a shared one together: decode's O = R + shared(X) + experts(X), and a training step whose
gradients of X meet in the shared expert's backward."""
import pytest

import dense_bounds as DB

pytestmark = pytest.mark.gpu


def _t():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _shared(d, m, seed):
    torch = _t()
    g = torch.Generator(device="cuda").manual_seed(seed)
    Wu = (torch.randn((d, 2 * m), generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    Wd = (torch.randn((m, d), generator=g, device="cuda") * m ** -0.5).to(torch.bfloat16)
    bu, bd = (torch.randn(s, generator=g, device="cuda") * 0.1 for s in (2 * m, d))
    return Wu, Wd, bu, bd


@pytest.mark.parametrize("T", [1, 11, 48])
def test_decode_step(T):
    torch = _t()
    from paper_2512_14080_amd import workloads as W
    from paper_2512_14080_amd.layer import DeviceLayer, SharedExpert
    cfg = W.MoEConfig("decode", T=T, d=256, n=128, E=16, K=4, m_tile=64)
    inp = W.make_inputs(cfg, 5, T=T)
    layer = DeviceLayer(inp)
    Wu, Wd, bu, bd = _shared(256, 200, 6)
    shared = SharedExpert(T, Wu, Wd, bu, bd)
    R = torch.randn((T, 256), device="cuda").to(torch.bfloat16)
    S = torch.empty_like(R)
    idx = torch.empty((T, 4), dtype=torch.int32, device="cuda")
    shared.forward(layer.X, S, R)
    layer.decode(S, topk_idx=idx)
    torch.cuda.synchronize()
    # the shared expert, its A rounded; its sum with R rounded; then the experts' bound at the kernel's own selection
    _, _, A, eA = DB.linear(layer.X, Wu, bu, None, "swiglu")
    ref = A @ Wd.double() + bd.double() + R.double()
    e = eA @ Wd.double().abs() + DB.E(200) * (A.abs() @ Wd.double().abs() + bd.double().abs()) + 2.0 ** -23 * ref.abs()
    e = e + DB.U * (ref.abs() + e)
    DB.within(S, ref, e, "shared")
    l = layer.X.double() @ layer.Wr.double()
    if layer.bias is not None:
        l = l + layer.bias.double()
    w = torch.softmax(torch.gather(l, 1, idx.long()), 1)
    ew = w * (2 * DB.E(256) * (layer.X.double().abs() @ layer.Wr.double().abs()).amax(1, keepdim=True) + DB.F)
    O, eO = DB.decode(layer.X, layer.W1, layer.W2, None, None, S, idx.long(), w, ew)
    DB.within(layer.O, O, eO, "O")


def test_training_step():
    """dX of the whole is the experts' dX, added in the shared expert's backward, in place."""
    torch = _t()
    from paper_2512_14080_amd import workloads as W
    from paper_2512_14080_amd.layer import DeviceLayer, SharedExpert
    T, d, m = 300, 256, 136
    cfg = W.MoEConfig("train", T=T, d=d, n=128, E=16, K=2, m_tile=64)
    layer = DeviceLayer(W.make_inputs(cfg, 7, T=T))
    Wu, Wd, bu, bd = _shared(d, m, 8)
    shared = SharedExpert(T, Wu, Wd, bu, bd, train=True)
    layer.step()
    Y = torch.empty_like(layer.O)
    shared.forward(layer.X, Y, layer.O)
    torch.cuda.synchronize()
    dX_experts = layer.dX.clone()
    shared.backward(layer.dO, layer.X, layer.dX, layer.dX)
    torch.cuda.synchronize()
    # the down-projection's gradients at the kept A, then the up-projection's at the kept H and the kernel's own dA
    down = DB.linear_grad(layer.dO, shared.A, Wd, None, None, "none")
    DB.within(shared.dA, *down["dX"], "dA")
    DB.within(shared.dWd, *down["dW"], "dWd")
    DB.within(shared.dbd, *down["db"], "dbd")
    up = DB.linear_grad(shared.dA, layer.X, Wu, shared.H, dX_experts, "swiglu")
    DB.within(layer.dX, *up["dX"], "dX")
    DB.within(shared.dWu, *up["dW"], "dWu")
    DB.within(shared.dbu, *up["db"], "dbu")
    _, _, y, ey = DB.linear(shared.A, Wd, bd, layer.O, "none")
    DB.within(Y, y, ey, "Y")


def test_refusals():
    torch = _t()
    from paper_2512_14080_amd.layer import SharedExpert
    Wu, Wd, _, _ = _shared(64, 40, 1)
    with pytest.raises(ValueError):
        SharedExpert(4, Wu, Wd[:32].contiguous())
    with pytest.raises(ValueError):
        SharedExpert(4, Wu[:, :72].contiguous(), Wd)
    assert torch.isfinite(Wu).all()
