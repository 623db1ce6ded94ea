"""GELU and SiLU of the 8-bit dense layer in fp32, on every route, where z itself is exact: what is
left is the activation's own arithmetic.

Bounds, with x = |z| / sqrt 2 (erff, expf, a power of two at most 2 ulp, a reciprocal 1, all else rounded
to nearest).  gelu: |z| / 2 (2^-23 x erf'(x) + 2^-22 erf(x) + 2^-24 (1 + erf(z / sqrt 2))), then one rounding.
- (z / 2) (1 + erf(z / sqrt 2)): the constant and its product are each off by at most 2^-24, which moves
  erf(x) by at most 2^-23 x erf'(x); erff 2 2^-23 |erf|; the sum 2^-24 (1 + erf).
- |z| < 1.5, z / 2 + z (z R): R is off by 2.7e-9 of it and the roundings of its last two steps, 2^-23 of it,
  z R by 2^-24 more; z^2 R is |z| / 2 erf(x), so that 2^-22 erf(x) covers them.
- beyond, max(z, 0) - |z| / 2 erfc(x): erfc is off by 6e-7 of it for the fit, 2^-22 and z^2 2^-24 for the
  exponential, 2 2^-23 for the reciprocal's part in both factors, 6 2^-24 for roundings: 1.5e-6 of 0.134 at
  1.5, 1.7e-6 of 0.046 at 2 and ever less, where 2^-22 erf(x) alone is 2.06e-7 and more.
silu = z / (1 + e^-z): e^-z is off by at most 2^-22 of it and two roundings (2^-23), 1 + e^-z by 2^-24, its
reciprocal by 2^-23; then one product.
"""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune
from test_gpu_finetune import _gen, _near, _no_timeouts, _normal
from test_gpu_int8 import _codes

pytestmark = pytest.mark.gpu
SHAPES = [(3, 70, 90), (9, 4096, 300), (40, 300, 4000), (300, 2048, 1000), (2000, 1500, 1500), (2000, 1500, 1501),
          (1999, 9216, 601)]


def _exact_z(shape, low):
    """(x, xscale, weight, wscale, z): sums of codes below 2^24 times powers of two; z below 60."""
    N, Cs, Ct = shape
    g = _gen(1)
    x, w = _codes(g, N, Cs), _codes(g, Ct, Cs)
    # (random sums are near 73^2 sqrt(Cs))
    top = math.ceil(math.log2(5400 * math.sqrt(Cs))) - 3
    ws = 2.0 ** -(top + torch.arange(Ct, device="cuda") % 12 + low).float()
    s = x.double() @ w.double().T
    assert float(s.abs().max()) < 2 ** 24
    z = s * ws.double()
    assert float(z.abs().max()) < 60
    return x, torch.ones(N, device="cuda"), w, ws, z


def _bound(z, act):
    if act == "silu":
        e = torch.exp(-z)
        return (z * torch.sigmoid(z)).abs() * ((2.0 ** -22 + 2.0 ** -23) * e / (1 + e) + 2.0 ** -24 + 2.0 ** -23)
    x = z.abs() / math.sqrt(2)
    slope = 2 / math.sqrt(math.pi) * torch.exp(-x * x)
    up = torch.special.erfc(-z / math.sqrt(2))
    return z.abs() / 2 * (2.0 ** -23 * x * slope + 2.0 ** -22 * torch.erf(x) + 2.0 ** -24 * up)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("low", [0, 8])
@pytest.mark.parametrize("shape", SHAPES)
def test_fp32_activations(shape, low, act):
    x, xs, w, ws, z = _exact_z(shape, low)
    y = q.int8_dense_forward(x, w, ws, act=act, xscale=xs)
    _near(y, plain_finetune.act(z, act), _bound(z, act))
    # the residual is one sum more
    r = _normal(_gen(2), *z.shape)
    assert torch.equal(q.int8_dense_forward(x, w, ws, act=act, xscale=xs, residual=r), y + r)
    _no_timeouts()
