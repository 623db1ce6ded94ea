"""Cross entropy whose gradient goes in pieces of the classes, on the GPU against its plain
64-bit form (tests/plain_finetune.py)."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_xent
from test_gpu_finetune import BF16, TYPES, _gen, _near, _no_timeouts, _normal, _xent_case, _xent_near

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_given_back():
    """The 64-bit forms take gigabytes, which other tests' measured memory does not have."""
    yield
    torch.cuda.empty_cache()


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


# Two to nine pieces, whose offsets are in the weights, the bias, the classes' numbers, dW and dbias, and
# whose dx is a sum over pieces; rows on 16 bytes and not, a last piece of odd width.
PIECES = [(1500, 40, 50001), (4100, 72, 40007), (9000, 33, 20003), (20000, 24, 4000), (3000, 520, 30011),
          (300, 64, 300001), (130000, 8, 700)]


def near(got, x, w, t, b=None, dloss=None):
    want, bound = plain_xent.xent(x, w, t, b, dloss)
    for a, c, e, n in zip(got, want, bound, ("loss", "lse", "dx", "dw", "db")):
        _near(a, c, e, n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,Cs,Ct", PIECES)
def test_several_pieces(N, Cs, Ct, dtype):
    r = q.xent_route(N, Cs, Ct, dtype)
    assert not r["kept"] and r["pieces"] > 1
    g, x, w, b, t = _xent_case(N, Cs, Ct, dtype, seed=34)
    # classes at both ends of each piece are some row's, and some are out
    ends = [c for i in range(r["pieces"]) for c in (i * r["piece"], min(Ct, (i + 1) * r["piece"]) - 1)]
    t[:len(ends)] = torch.tensor(ends, device="cuda")
    t[len(ends)::11] = -100
    b[r["piece"] + 1] = -math.inf
    t[t == r["piece"] + 1] = 0
    near(q.xent_grad(x, w, t, b), x, w, t, b)
    dloss = torch.randn(N, generator=g, device="cuda")
    near(q.xent_grad(x, w, t, dloss=dloss), x, w, t, None, dloss)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 1)])
def test_pieces_of_strided_matrices(pad, off, dtype):
    N, Cs, Ct = 4100, 36, 40007
    assert q.xent_route(N, Cs, Ct, dtype)["pieces"] > 1
    g = _gen(35)
    x = _normal(g, N, Cs, dtype=dtype, pad=pad, off=off)
    w = _normal(g, Ct, Cs, dtype=dtype, scale=2 / math.sqrt(Cs), pad=pad, off=off)
    t = torch.randint(0, Ct, (N,), generator=g, device="cuda")
    got = q.xent_grad(x, w, t)
    near(got, x, w, t)
    assert all(torch.equal(a, c) for a, c in zip(got, q.xent_grad(x, w, t)))
