"""Cross entropy with classes masked by the lowest finite value, kept logits and not, against the
64-bit form whose bounds leave masked classes out (tests/plain_xent.py)."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_xent
from test_gpu_finetune import BF16, F32, TYPES, _near, _no_timeouts, _xent_case

pytestmark = pytest.mark.gpu


def near(got, x, w, t, b=None, dloss=None):
    want, bound = plain_xent.xent(x, w, t, b, dloss)
    for e in bound[:2]:
        assert float(e.max()) < 1e-2  # (a bound that says something)
    for a, c, e, n in zip(got, want, bound, ("loss", "lse", "dx", "dw", "db")):
        _near(a, c, e, n)


# (kept in both calls, in one of them, in none)
SIZES = [(5, 48, 70), (120, 64, 1000), (1000, 40, 5000), (512, 96, 4100), (600, 40, 30001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lowest", [F32, BF16, None])
@pytest.mark.parametrize("where", ["first", "last", "both", "ends of tiles"])
@pytest.mark.parametrize("N,Cs,Ct", SIZES)
def test_masked_by_the_lowest_value(N, Cs, Ct, where, lowest, dtype):
    """The first half of the classes, the last, a band in the middle left, or all but a few: blocks
    of 16 columns and whole tiles of them masked, before and after others."""
    _, x, w, b, t = _xent_case(N, Cs, Ct, dtype, seed=32)
    out = torch.zeros(Ct, dtype=torch.bool, device="cuda")
    if where in ("first", "both"):
        out[:Ct // 2 if where == "first" else Ct // 3] = True
    if where in ("last", "both"):
        out[Ct // 2 if where == "last" else Ct - Ct // 3:] = True
    if where == "ends of tiles":
        out[:] = True
        out[15::64] = False
    b[out] = -math.inf if lowest is None else torch.finfo(lowest).min
    inside = (~out).nonzero()[:, 0]
    t = inside[t % inside.numel()].contiguous()
    t[N // 2] = -100
    near(q.xent_forward(x, w, t, b), x, w, t, b)
    got = q.xent_grad(x, w, t, b)
    near(got, x, w, t, b)
    assert not got[3][out].any() and not got[4][out].any()  # no gradient to what is masked
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,Cs,Ct", SIZES)
def test_every_class_at_the_lowest_value(N, Cs, Ct, dtype):
    """All logits are the lowest value then (what the products add to it is less than half of its
    last bit): lse is that value as well, and nothing is NaN or infinite."""
    _, x, w, b, t = _xent_case(N, Cs, Ct, dtype, seed=33)
    b[:] = torch.finfo(F32).min
    got = q.xent_grad(x, w, t, b)
    assert bool((got[1] == torch.finfo(F32).min).all())
    assert all(bool(torch.isfinite(v).all()) for v in got)
