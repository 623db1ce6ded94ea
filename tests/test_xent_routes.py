"""How cross entropy goes about its sizes, by the host-side route query."""
import ctypes
import math
import random

import pytest
import torch

import paper_1512_06473_gb300 as q
from paper_1512_06473_gb300 import _lib

F32, BF16 = torch.float32, torch.bfloat16


def _sizes():
    # narrow layers of many rows and classes, where a tile of dx is shared by CTAs
    named = [(16384, 128, 50257), (8192, 128, 128256), (4096, 128, 145161), (8192, 256, 256000),
             (4096, 128, 256000), (8192, 128, 100277)]
    r = random.Random(11)
    drawn = [tuple(int(2 ** r.uniform(*span)) for span in ((0, 15), (3, 12), (3, 18))) for _ in range(1500)]
    return named + [s for s in drawn if math.prod(s) < 2 ** 42]


def test_every_share_of_dx_has_classes():
    """A CTA without terms would leave its part of the sum unwritten: the last piece of
    the classes is shorter than the others, and shared by no more CTAs than it has blocks."""
    several = shared = 0
    for N, Cs, Ct in _sizes():
        for dtype in (F32, BF16):
            r = q.xent_route(N, Cs, Ct, dtype)
            assert (r["pieces"] - 1) * r["piece"] + r["last"] == Ct and 0 < r["last"] <= r["piece"]
            assert r["shares"] >= 1
            assert (r["shares"] - 1) * r["share_classes"] < r["last"], (N, Cs, Ct, dtype, r)
            assert r["shares"] * r["share_classes"] >= r["last"], (N, Cs, Ct, dtype, r)
            several += r["pieces"] > 1
            shared += r["pieces"] > 1 and r["shares"] > 1
    assert several > 100 and shared > 20


def test_kept_logits_are_one_piece():
    r = q.xent_route(128, 4096, 1000)
    assert r["kept"] and r["pieces"] == 1 and r["piece"] == r["last"] == 1000
    r = q.xent_route(128, 4096, 1000, grad=False)
    assert r["kept"] and r["shares"] == r["share_classes"] == 0
    assert not q.xent_route(4096, 2048, 32768, BF16)["kept"]


@pytest.mark.parametrize("bad", [(0, 8, 8, 0), (8, 0, 8, 0), (8, 8, 0, 0), (8, 8, 8, 2), (-1, 8, 8, 1)])
def test_the_query_refuses(bad):
    info = (ctypes.c_int * 6)()
    assert q.load().qcnn_xent_route_info(*bad, 1, info) == _lib.ERR_INVALID_ARG
    assert q.load().qcnn_xent_route_info(8, 8, 8, 0, 1, None) == _lib.ERR_INVALID_ARG
    with pytest.raises(TypeError):
        q.xent_route(8, 8, 8, torch.float16)
