"""Orthogonalising matrices of tiny and of large values with eps 0: the norm is that of the matrix,
in the form of one launch and as products."""
import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune as plain
from test_gpu_finetune import BF16, F32, TYPES, _gen, _no_timeouts, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("exponent", [-140, -120, -100, -70, -62, -49, -47, 40, 60, 110])
@pytest.mark.parametrize("shape", [(40, 64), (100, 130), (300, 150), (129, 2100)])
def test_scales_without_eps(shape, exponent, dtype):
    """As test_gpu_finetune's bound; -140: subnormal values, taken as they are."""
    m, n = shape
    g = (_normal(_gen(51), m, n) * 2.0 ** exponent).to(dtype)
    g[0, 0] = 2.0 ** (exponent - 9)
    want = plain.orthogonalize(g, eps=0)
    unit = 2.0 ** -24 if dtype == F32 else 2.0 ** -17
    sums = (32 + max(m, n) / (16 if dtype == BF16 else 64)) * 2.0 ** -23
    limit = 485 * (unit + sums) * 3 + plain.eps_out(dtype) * float(want.norm())
    assert float((q.orthogonalize(g, eps=0).double() - want).norm()) <= limit
    # before any step: the matrix by its norm (eight squares of a lane, 2^-24 each of their sum, half of
    # that of the root; the factor and the product, 2^-24 each)
    want = plain.orthogonalize(g, 0, eps=0)
    got = q.orthogonalize(g, 0, eps=0).double()
    assert float((got - want).norm()) <= 2.0 ** -21 + plain.eps_out(dtype)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
def test_values_far_apart(dtype):
    """Tiny, ordinary and large values in one matrix: each squared where it neither overflows nor
    vanishes."""
    for exponents in ((-100, -60), (-60, -30), (-30, 0), (0, 49), (30, 80)):
        g = torch.zeros(100, 130, device="cuda")
        g[:50] = torch.randn(50, 130, generator=_gen(52), device="cuda") * 2.0 ** exponents[0]
        g[50] = torch.randn(130, generator=_gen(53), device="cuda") * 2.0 ** exponents[1]
        g = g.to(dtype)
        want = plain.orthogonalize(g, 0, eps=0)
        got = q.orthogonalize(g, 0, eps=0).double()
        assert float((got - want).norm()) <= 2.0 ** -21 + plain.eps_out(dtype)
