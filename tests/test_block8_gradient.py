"""What the backward from an 8-bit checkpoint is after the 8-bit forward: the 16-bit layer's at that forward's H, which the
gradient with every rounding passed straight through comes near, and equals where nothing is rounded."""
import numpy as np
import pytest
import torch

import oracle
from oracle import block8


def _straight_through(X, W1, W2, Wr, member, dO):
    """Gradients of the 8-bit forward by torch's autograd, every rounding passed straight through."""
    x, w1, w2, wr = (torch.tensor(a, requires_grad=True) for a in (X, W1, W2, Wr))

    def through(v, q):
        return v + (torch.tensor(q) - v).detach()

    n = W2.shape[1]
    x8 = through(x, block8.through(X))
    q1, q2 = (through(w, q) for w, q in zip((w1, w2), block8.through_experts(W1, W2)))
    s = torch.softmax(x @ wr, 1) * torch.tensor(member.astype(np.float64))
    s = s / s.sum(1, keepdim=True)
    O = 0
    for e in range(W1.shape[0]):
        H = x8 @ q1[e]
        a = torch.nn.functional.silu(H[:, :n]) * H[:, n:]
        O = O + s[:, e:e + 1] * (through(a, block8.through(a.detach().numpy())) @ q2[e])
    (O * torch.tensor(dO)).sum().backward()
    return {"dX": x.grad.numpy(), "dW1": w1.grad.numpy(), "dW2": w2.grad.numpy(), "dWr": wr.grad.numpy()}


def _off(a, b):
    return {k: np.linalg.norm(a[k] - b[k]) / np.linalg.norm(b[k]) for k in b}


def _layer(rng, T, d, n, E, K):
    X, dO = rng.standard_normal((T, d)), rng.standard_normal((T, d))
    W1, W2 = rng.standard_normal((E, d, 2 * n)) * 0.04, rng.standard_normal((E, n, d)) * 0.04
    Wr = rng.standard_normal((d, E)) * d ** -0.5
    S = oracle.softmax_scores(X @ Wr)
    member = oracle.tc_membership(oracle.topk_select(S.astype(np.float32), K), E)
    return X, W1, W2, Wr, dO, member, oracle.routing_from_membership(member, S, np.float64)


@pytest.mark.parametrize("seed", [0, 1])
def test_distance_to_the_straight_through_gradient(seed):
    X, W1, W2, Wr, dO, member, R = _layer(np.random.default_rng(seed), 128, 256, 192, 8, 2)
    fw = block8.forward_quant(X, W1, W2, R)
    H = block8.through_halves(fw["H"])
    want = _straight_through(X, W1, W2, Wr, member, dO)
    W1q, W2q = block8.through_experts(W1, W2)
    # A rounding is at most 2^-4 of a value off, 2^-4 / sqrt 3 in the root mean square; a gradient's product is through at most
    # six that only one of the two has (X, W1, W2, A, and the kept gate and up).
    most = 2.0 ** -4 / 3 ** 0.5 * 6 ** 0.5
    for x, w1, w2 in ((X, W1, W2), (fw["X8"], W1, W2), (fw["X8"], W1q, W2q)):
        off = _off(block8.backward_ckpt(dO, x, H, w1, w2, Wr, R), want)
        print({k: f"{v:.4f}" for k, v in off.items()})
        assert 0.01 < min(off.values()) and max(off.values()) < most, off


def test_it_is_that_gradient_where_nothing_is_rounded(monkeypatch):
    X, W1, W2, Wr, dO, member, R = _layer(np.random.default_rng(2), 16, 128, 64, 8, 2)
    monkeypatch.setattr(block8, "through", lambda x, block=None: np.asarray(x, np.float64))
    H = block8.forward_quant(X, W1, W2, R)["H"]
    off = _off(block8.backward_ckpt(dO, X, H, W1, W2, Wr, R), _straight_through(X, W1, W2, Wr, member, dO))
    assert max(off.values()) < 1e-12, off
