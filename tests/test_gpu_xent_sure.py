"""Rows that a network is sure of: one logit far above the others.  The inputs are whole numbers
small enough for every logit to be exact, so that only the softmax's own roundings are left."""
import pytest
import torch

import paper_1512_06473_gb300 as q
from test_gpu_finetune import BF16, F32, TYPES, _no_timeouts

pytestmark = pytest.mark.gpu


def _case(N, Ct, top, second, dtype):
    """Row n: class c_n has the logit `top`, class c_n + 17 (of Ct) `second`, all others 0; dx and
    dW's sums have one or two terms that are not 0 or far below it."""
    Cs = 64
    g = torch.Generator(device="cuda").manual_seed(41)
    c = torch.randint(0, Ct, (N,), generator=g, device="cuda")
    row = torch.arange(N, device="cuda")
    x, w = torch.zeros(N, Cs, dtype=dtype, device="cuda"), torch.zeros(Ct, Cs, dtype=dtype, device="cuda")
    # rows of one kind k = n mod 32 share their classes
    k = row % 32
    c = c[:32][k]
    x[row, k] = 1
    kinds = torch.arange(32, device="cuda")
    w[(c[:32] + 17) % Ct, kinds] = second
    w[c[:32], kinds] = top
    return x, w, c


# Kept and not, one tile of classes to many.  (top, second): the rest of the sum below half of fp32's
# last bit of 1, and above it.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,Ct", [(40, 200), (300, 2048), (700, 30001)])
@pytest.mark.parametrize("top,second", [(30, 0), (88, 80), (100, 96), (300, 295), (1000, 988)])
def test_sure_rows(N, Ct, top, second, dtype):
    """loss = log(1 + r) with r = exp(second - top) + ..., all other terms below 2^-42 of the sum or
    zero: r within (2^-22 + 3 * 2^-24 (top - second)) of itself, and 2^-24 each where it is added to 1
    (in its 16 columns, with another 16's, of lanes, warps and tiles: 12 times at most, with 0 or a
    power of two below it otherwise), log 2^-23 of itself; the gradient as near."""
    x, w, c = _case(N, Ct, top, second, dtype)
    l = x.double() @ w.double().T
    lse = torch.logsumexp(l, 1)
    # (log of the sum without the cancellation of lse - top)
    others = torch.exp(l - top).scatter(1, c[:, None], 0.0).sum(1)
    loss = torch.log1p(others)
    p = torch.exp(l - top) / (1 + others)[:, None]
    limit = others * (2.0 ** -22 + 3 * 2.0 ** -24 * (top - second) + 2.0 ** -23) + 12 * 2.0 ** -24
    got_loss, got_lse = q.xent_forward(x, w, c)
    again, _, dx, dw, db = q.xent_grad(x, w, c)
    for v in (got_loss, again):
        assert bool((v >= 0).all())
        assert bool(((v.double() - loss).abs() <= limit).all()), float((v.double() - loss).abs().max())
    assert bool(((got_lse.double() - lse).abs() <= limit + 2.0 ** -23 * top).all())
    # db: the sum over rows of (p - [target]) / N, each p within limit's and 2^-21 of itself
    near = (limit[:, None] * p + p * 2.0 ** -21 * (1 + (l - top).abs() * (p > 0))).sum(0) + N * 2.0 ** -24
    want = p.scatter_add(1, c[:, None], -torch.ones_like(lse)[:, None]).sum(0)
    assert bool(((db.double() * N - want).abs() <= near + N * 2.0 ** -24 * want.abs()).all())
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
    _no_timeouts()
