"""Products of long rows that the call itself quantizes, by pairs of CTAs: these drain a sum where the
magnitudes of x's codes, which the pass that makes the codes adds up, could leave 2^24.  Rows of one
magnitude have codes of +-127, and weights whose sums go far beyond 2^24 on the way and cancel to an
odd rest."""
import pytest
import torch

import paper_1512_06473_gb300 as q
from test_gpu_finetune import _gen, _no_timeouts
from test_gpu_int8 import _codes

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# every width of the quantizing pass's groups of threads, in both types
SHAPES = [(2000, 1030, 1500), (1999, 2047, 1535), (1999, 3000, 1535), (1999, 5001, 1535), (1999, 9216, 2001),
          (3000, 12003, 1501), (2304, 24001, 2048)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("shape", SHAPES)
def test_sums_of_rows_that_the_call_quantizes(shape, pad, off, dtype):
    N, Cs, Ct = shape
    assert q.int8_route(N, Cs, Ct)["ctas"] == 2
    g = _gen(1)
    half = (Cs - 11) // 2
    w = _codes(g, Ct, Cs, 100, 127)
    w[:, half:2 * half] = -w[:, :half]
    w[:, :half][torch.rand(Ct, half, generator=g, device="cuda") < 0.01] = -128
    room = torch.ones(N * (Cs + pad) + off, device="cuda")
    x = room.to(dtype)[off:].view(N, Cs + pad)[:, :Cs]
    x[1::3] *= -1
    x[2::3, 1::7] = 0
    x[N // 2:] *= 0.5
    codes, xs = q.int8_quantize(x)
    assert bool(((codes == 127) | (codes == -127) | (codes == 0)).all())
    one = torch.ones(Ct, device="cuda")
    want = codes.double() @ w.double().T
    assert float(want.abs().max()) < 2 ** 31 and bool((want % 2 == 1).any())
    # (a sum rounded to fp32 once, one product)
    want = want.float() * xs[:, None]
    y = q.int8_dense_forward(x, w, one, dtype=dtype)
    assert torch.equal(y, want.to(dtype))
    assert torch.equal(q.int8_dense_forward(codes, w, one, xscale=xs, dtype=dtype), y)
    _no_timeouts()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_long_row_among_short_ones(dtype):
    """Of a tile's rows the one with the largest magnitudes decides, wherever it lies."""
    N, Cs, Ct = 1999, 5001, 1535
    g = _gen(2)
    half = (Cs - 11) // 2
    w = _codes(g, Ct, Cs, 100, 127)
    w[:, half:2 * half] = -w[:, :half]
    one = torch.ones(Ct, device="cuda")
    x = torch.zeros(N, Cs, device="cuda", dtype=dtype)
    x[:, ::50] = 1
    for row in (0, 159, 160, 700, N - 1):
        x[row] = 1
    codes, xs = q.int8_quantize(x)
    want = (codes.double() @ w.double().T).float() * xs[:, None]
    assert torch.equal(q.int8_dense_forward(x, w, one), want.to(dtype))
