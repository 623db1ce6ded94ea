"""fp32 operands up to the largest finite value: bf16 rounds what is above 3.39e38 to infinity, the
sum of an operand's pieces does not."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune as plain
from test_gpu_finetune import BF16, F32, _gen, _near, _no_timeouts, _normal

pytestmark = pytest.mark.gpu
MOST = torch.finfo(F32).max


# few rows; weights split on their way, on 16 bytes and off; planes of both
@pytest.mark.parametrize("N,Cs,Ct", [(3, 96, 40), (40, 96, 64), (40, 97, 300), (300, 128, 130), (2000, 520, 700)])
def test_largest_operands(N, Cs, Ct):
    g = _gen(61)
    x, w = _normal(g, N, Cs), _normal(g, Ct, Cs, scale=1e-30)
    x[1, 5], x[0, Cs - 1], x[N - 1, 7] = MOST, -MOST, 3.4e38
    w[:, 7] = 0  # the lowest value in a place that nothing is taken from
    want, _, ey, _ = plain.dense_forward(x, w)
    _near(q.dense_forward(x, w), want, ey)
    v = _normal(g, Ct, Cs)
    v[2, 3], v[Ct - 1, 0] = -MOST, 3.4e38
    y = x.clamp(-5, 5) * 1e-30
    want, _, ey, _ = plain.dense_forward(y, v)
    _near(q.dense_forward(y, v), want, ey)
    dy = _normal(g, N, Ct, scale=1e-30)
    got = q.dense_backward(dy, y, v)
    want, bound = plain.dense_backward(dy, y, v)
    _near(got[0], want[0], bound[0], "dx")
    dy = _normal(g, N, Ct)
    dy[1, 1] = MOST
    want, bound = plain.dense_backward(dy, y, w)
    got = q.dense_backward(dy, y, w)
    for a, c, e, n in zip(got[:2], want, bound, ("dx", "dw")):
        _near(a, c, e, n)
    _no_timeouts()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_stay_non_finite(dtype):
    """What is infinite, or rounds to an infinite bf16 result, does not come out finite."""
    g = _gen(62)
    x, w = _normal(g, 40, 100, dtype=dtype), _normal(g, 48, 100, dtype=dtype)
    x[3, 7], w[5, 0] = math.inf, -math.inf
    bad = torch.zeros(40, 48, dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 5] = True
    assert torch.equal(~torch.isfinite(q.dense_forward(x, w)), bad)
    assert not torch.isfinite(q.dense_forward(x[:, 1:], w[:, 1:])[3]).any()  # (copied: off 16 bytes)
    dy = _normal(g, 40, 48, dtype=dtype)
    dy[9, 2] = math.inf
    dx, dw, db = q.dense_backward(dy, x[:, 8:], w[:, 8:], _normal(g, 40, 48, dtype=dtype), "silu")
    assert not torch.isfinite(dx[9]).any() and not torch.isfinite(dw[2]).any() and not math.isfinite(db[2])
    assert bool(torch.isfinite(dx[:9]).all()) and bool(torch.isfinite(dw[3:]).all())
    t = torch.randint(0, 48, (40,), generator=g, device="cuda")
    t[3] = -100
    dloss = torch.ones(40, device="cuda")
    dloss[11] = math.inf
    w[5, 0] = 0
    _, _, dx, dw, db = q.xent_grad(x, w, t, dloss=dloss)
    assert not torch.isfinite(dx[11]).any() and not torch.isfinite(db).any()
    assert bool(torch.isfinite(dx[:3]).all()) and not dx[3].any()
