"""The plain forms that the GPU tests of the fine-tuning operators are held to: their
gradients against central differences of their own values, and against torch's autograd."""
import pytest
import torch

import plain_finetune as plain

torch.manual_seed(0)


def _t(*shape, scale=1.0):
    return torch.randn(*shape, dtype=torch.float64) * scale


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_dense_gradients_are_the_values_differences(name):
    x, w, b, dy = _t(7, 5), _t(4, 5), _t(4), _t(7, 4)
    z = x @ w.T + b
    (dx, dw, db), _ = plain.dense_backward(dy, x, w, z, name)

    def value(x, w, b):
        return float((plain.act(x @ w.T + b, name) * dy).sum())

    h = 1e-6
    for grad, arg in ((dx, 0), (dw, 1), (db, 2)):
        args = [x, w, b]
        v = torch.randn_like(args[arg])
        up, down = list(args), list(args)
        up[arg], down[arg] = args[arg] + h * v, args[arg] - h * v
        diff = (value(*up) - value(*down)) / (2 * h)
        # central differences: third derivatives h^2, and 2^-52 |value| / h of cancellation
        assert abs(diff - float((grad * v).sum())) < 1e-6


@pytest.mark.parametrize("weights", [False, True])
def test_xent_gradients_are_the_values_differences(weights):
    x, w, b = _t(6, 5), _t(9, 5), _t(9)
    t = torch.tensor([0, 8, -100, 3, 3, 9])  # one ignored, one out of range
    dloss = torch.rand(6, dtype=torch.float64) if weights else None
    (loss, lse, dx, dw, db), _ = plain.xent(x, w, t, b, dloss)
    keep = (t >= 0) & (t < 9)
    assert torch.equal(loss[~keep], torch.zeros(2, dtype=torch.float64))
    g = dloss if weights else torch.full((6,), 0.25, dtype=torch.float64)

    def value(x, w, b):
        return float((plain.xent(x, w, t, b, dloss)[0][0] * g).sum())

    h = 1e-6
    for grad, arg in ((dx, 0), (dw, 1), (db, 2)):
        args = [x, w, b]
        v = torch.randn_like(args[arg])
        up, down = list(args), list(args)
        up[arg], down[arg] = args[arg] + h * v, args[arg] - h * v
        diff = (value(*up) - value(*down)) / (2 * h)
        assert abs(diff - float((grad * v).sum())) < 1e-6


def test_xent_is_torchs():
    x, w, b = _t(6, 5).requires_grad_(), _t(9, 5).requires_grad_(), _t(9).requires_grad_()
    t = torch.tensor([0, 8, -100, 3, 3, 1])
    want = torch.nn.functional.cross_entropy(x @ w.T + b, t)
    want.backward()
    (loss, _, dx, dw, db), _ = plain.xent(x.detach(), w.detach(), t, b.detach())
    assert abs(float(loss.sum() / 5 - want)) < 1e-12
    for got, ref in ((dx, x), (dw, w), (db, b)):
        assert torch.allclose(got, ref.grad, atol=1e-12)


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6)])
def test_newton_schulz_moves_singular_values_only(shape):
    """The polynomial acts on the singular values alone: U p(S) V^T."""
    g = _t(*shape)
    u, s, vt = torch.linalg.svd(g, full_matrices=False)
    s = s / (torch.linalg.vector_norm(g) + 1e-7)
    a, b, c = plain.NS
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert torch.allclose(plain.orthogonalize(g), (u * s) @ vt, atol=1e-9)
