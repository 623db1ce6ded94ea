"""Scales of the 8-bit dense layer at both ends of fp32's range: their product with a sum, and each of
its two steps, may leave the range only where the result does."""
import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _no_timeouts, _normal
from test_gpu_int8 import _codes

pytestmark = pytest.mark.gpu
SHAPES = [(2, 300, 40), (70, 300, 4000), (300, 2048, 1000), (2000, 1500, 1500), (2000, 1500, 1501)]
TOP = torch.finfo(torch.float32).max


def _check(y, want, bound):
    """As _near, but infinite where the result is beyond fp32's range."""
    beyond = want.abs() > TOP * (1 + 2.0 ** -20)
    sure = want.abs() < TOP * (1 - 2.0 ** -20)
    assert torch.equal(y.double()[beyond], torch.sign(want[beyond]) * float("inf"))
    _near(torch.where(sure, y, torch.zeros_like(y)), torch.where(sure, want, torch.zeros_like(want)),
          torch.where(sure, bound, torch.zeros_like(bound)))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pair", [(1e36, 1e-36), (1e-36, 1e36), (2.0 ** 96, 2.0 ** -96), (3e38, 2.0 ** -126),
                                  (2.0 ** -126, 3e38), (1e36, 1e-3), (2.0 ** 100, 2.0 ** 100)])
def test_one_large_and_one_small(shape, pair):
    N, Cs, Ct = shape
    g = _gen(1)
    x, w = _codes(g, N, Cs), _codes(g, Ct, Cs)
    x[0] = 0  # (sums of zero stay zero)
    xs, ws = torch.full((N,), pair[0], device="cuda"), torch.full((Ct,), pair[1], device="cuda")
    y = q.int8_dense_forward(x, w, ws, xscale=xs)
    _check(y, *plain.dense(x, xs, w, ws))
    assert bool((y[0] == 0).all())
    _no_timeouts()


@pytest.mark.parametrize("shape", SHAPES)
def test_rows_and_outputs_of_every_size(shape):
    N, Cs, Ct = shape
    g = _gen(2)
    x, w = _codes(g, N, Cs), _codes(g, Ct, Cs)
    xs = 2.0 ** (torch.randint(-126, 128, (N,), generator=g, device="cuda").double())
    ws = 2.0 ** (torch.randint(-126, 128, (Ct,), generator=g, device="cuda").double())
    xs, ws = xs.float() * 1.25, ws.float() * 1.125
    b = torch.randn(Ct, generator=g, device="cuda")
    assert bool(torch.isfinite(xs).all()) and bool(torch.isfinite(ws).all())
    _check(q.int8_dense_forward(x, w, ws, xscale=xs), *plain.dense(x, xs, w, ws))
    _check(q.int8_dense_forward(x, w, ws, b, xscale=xs), *plain.dense(x, xs, w, ws, b))


@pytest.mark.parametrize("shape", SHAPES)
def test_large_activations(shape):
    N, Cs, Ct = shape
    g = _gen(3)
    x = _normal(g, N, Cs, scale=2e37)
    w, ws = _codes(g, Ct, Cs), torch.full((Ct,), 1e-5, device="cuda")
    c, s = plain.quantize(x)
    want, bound = plain.dense(c.cuda(), s.cuda(), w, ws)
    assert float(s.max()) > 2.0 ** 96 and float(want.abs().max()) < TOP
    _near(q.int8_dense_forward(x, w, ws), want, bound)
