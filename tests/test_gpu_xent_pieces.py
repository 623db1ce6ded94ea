"""Cross entropy whose gradient goes in pieces of the classes, on the GPU against its plain
64-bit form (tests/plain_finetune.py)."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
from test_gpu_finetune import BF16, _no_timeouts, _xent_case, _xent_near

pytestmark = pytest.mark.gpu


# Pieces whose dx is shared by two, four or eight CTAs, the last one too short for as many (on how
# many depends on the clusters that the device holds at once).
@pytest.mark.parametrize("N,Cs,Ct", [(17949, 100, 21524), (4096, 128, 145161)])
def test_a_short_last_piece(N, Cs, Ct):
    r = q.xent_route(N, Cs, Ct, BF16)
    assert not r["kept"] and r["pieces"] > 1 and r["last"] < r["piece"]
    assert q.xent_route(N, Cs, r["piece"] * r["pieces"], BF16)["shares"] > 1
    _, x, w, b, t = _xent_case(N, Cs, Ct, BF16, seed=31)
    t[::7] = -100
    b[Ct // 3] = -math.inf
    t[t == Ct // 3] = 0
    _xent_near(q.xent_grad(x, w, t, b), x, w, t, b)
    _no_timeouts()
