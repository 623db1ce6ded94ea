"""Argument checks and workspace queries of the fine-tuning entry points: host-side, no
kernel is launched."""
import ctypes

import pytest
import torch

import paper_1512_06473_gb300 as q
from paper_1512_06473_gb300 import _lib

lib = _lib.load()
F32, BF16 = _lib.F32, _lib.BF16
P = 256  # a pointer that is aligned and never followed


def _bytes(query, *args):
    nb = ctypes.c_size_t()
    assert getattr(lib, query)(*args, ctypes.byref(nb)) == _lib.OK
    return nb.value


def _forward(N=16, Cs=64, Ct=32, x=P, ldx=64, W=P, ldw=64, bias=None, act=0, r=None, ldr=0, y=P, ldy=32,
             pre=None, ldp=0, dtype=F32, ws=P, wsb=0):
    return lib.qcnn_dense_forward(x, ldx, N, Cs, W, ldw, Ct, bias, act, r, ldr, y, ldy, pre, ldp, dtype, ws,
                                  wsb, None)


@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(Cs=0), dict(Ct=0), dict(dtype=2), dict(act=4), dict(act=-1), dict(x=None), dict(W=None),
    dict(y=None), dict(ldx=63), dict(ldw=63), dict(ldy=31), dict(x=P + 2), dict(W=P + 1), dict(y=P + 2),
    dict(bias=P + 2), dict(r=P, ldr=31), dict(r=P + 1, ldr=32), dict(pre=P, ldp=31),
    dict(dtype=BF16, x=P + 1)])
def test_dense_forward_refuses(bad):
    assert _forward(**bad) == _lib.ERR_INVALID_ARG


def test_dense_forward_wants_its_workspace():
    need = _bytes("qcnn_dense_forward_workspace_size", 16, 64, 32, F32, 1)
    assert need > 0
    assert _forward(wsb=need - 1) == _lib.ERR_WORKSPACE
    assert _forward(ws=None, wsb=need) == _lib.ERR_WORKSPACE
    assert _forward(ws=P + 128, wsb=need) == _lib.ERR_WORKSPACE


def test_nothing_to_do_is_done():
    assert _forward(N=0, x=None, y=None) == _lib.OK
    assert lib.qcnn_xent_forward(None, 8, 0, 8, P, 8, 4, None, None, None, None, F32, None, 0, None) == _lib.OK


def test_workspaces():
    # few rows need none, aligned bf16 only what split sums take
    for dtype in (F32, BF16):
        assert _bytes("qcnn_dense_forward_workspace_size", 8, 4096, 1000, dtype, 1) == 0
        assert _bytes("qcnn_dense_forward_workspace_size", 0, 64, 64, dtype, 1) == 0
    assert _bytes("qcnn_dense_forward_workspace_size", 4096, 4096, 4096, BF16, 1) == 0
    assert _bytes("qcnn_dense_forward_workspace_size", 4096, 4096, 4096, BF16, 0) >= 2 * 2 * 4096 * 4096
    # cross entropy of many classes: a bounded piece of the logits' gradient
    logits = 4 * 4096 * 200000
    got = _bytes("qcnn_xent_workspace_size", 4096, 1024, 200000, BF16, 1, 1)
    assert got < logits / 8
    assert _bytes("qcnn_xent_workspace_size", 4096, 1024, 200000, BF16, 1, 0) < logits / 16
    for query, n in (("qcnn_dense_forward_workspace_size", 5), ("qcnn_dense_backward_workspace_size", 5),
                     ("qcnn_xent_workspace_size", 6), ("qcnn_orthogonalize_workspace_size", 3)):
        assert getattr(lib, query)(*([1] * n), None) == _lib.ERR_INVALID_ARG
        nb = ctypes.c_size_t()
        assert getattr(lib, query)(-1, *([1] * (n - 1)), ctypes.byref(nb)) == _lib.ERR_INVALID_ARG


def _backward(N=16, Cs=64, Ct=32, dy=P, lddy=32, x=P, ldx=64, W=P, ldw=64, pre=P, ldp=32, act=1, dx=P, lddx=64,
              dW=P, lddw=64, db=P, dtype=F32, ws=P, wsb=0):
    return lib.qcnn_dense_backward(dy, lddy, x, ldx, W, ldw, pre, ldp, N, Cs, Ct, act, dx, lddx, dW, lddw, db,
                                   dtype, ws, wsb, None)


@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(Cs=0), dict(Ct=0), dict(dtype=-1), dict(act=9), dict(dy=None), dict(lddy=31), dict(x=None),
    dict(W=None), dict(pre=None), dict(ldp=31), dict(lddx=63), dict(lddw=63), dict(dx=P + 2), dict(dW=P + 2),
    dict(db=P + 2)])
def test_dense_backward_refuses(bad):
    assert _backward(**bad) == _lib.ERR_INVALID_ARG


def test_dense_backward_needs_only_what_it_reads():
    # (no workspace is given: the next check after the arguments')
    assert _backward(dW=None, x=None, ldx=0) == _lib.ERR_WORKSPACE
    assert _backward(dx=None, W=None, ldw=0) == _lib.ERR_WORKSPACE
    assert _backward(act=0, pre=None, ldp=0) == _lib.ERR_WORKSPACE


def _xent(grad=False, N=16, Cs=64, Ct=32, x=P, ldx=64, W=P, ldw=64, bias=None, t=P, dloss=None, loss=P, lse=P,
          dx=P, lddx=64, dW=P, lddw=64, db=None, dtype=F32, ws=None, wsb=0):
    if grad:
        return lib.qcnn_xent_grad(x, ldx, N, Cs, W, ldw, Ct, bias, t, dloss, loss, lse, dx, lddx, dW, lddw, db,
                                  dtype, ws, wsb, None)
    return lib.qcnn_xent_forward(x, ldx, N, Cs, W, ldw, Ct, bias, t, loss, lse, dtype, ws, wsb, None)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(Cs=0), dict(Ct=0), dict(dtype=7), dict(x=None), dict(W=None), dict(t=None), dict(t=P + 4),
    dict(loss=None), dict(lse=None), dict(ldx=63), dict(ldw=63), dict(bias=P + 1), dict(loss=P + 2)])
def test_xent_refuses(grad, bad):
    assert _xent(grad, **bad) == _lib.ERR_INVALID_ARG
    assert _xent(grad) == _lib.ERR_WORKSPACE


@pytest.mark.parametrize("bad", [dict(dx=None), dict(dW=None), dict(lddx=63), dict(lddw=63), dict(dloss=P + 2),
                                 dict(db=P + 1)])
def test_xent_grad_refuses(bad):
    assert _xent(True, **bad) == _lib.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(m=0), dict(n=0), dict(steps=-1), dict(steps=101), dict(eps=-1.0), dict(eps=float("nan")), dict(G=None),
    dict(out=None), dict(ldg=31), dict(ldo=31), dict(dtype=2), dict(G=P + 2)])
def test_orthogonalize_refuses(bad):
    a = dict(G=P, ldg=32, m=16, n=32, steps=5, eps=0.0, out=P, ldo=32, dtype=F32)

    def call(a):
        return lib.qcnn_orthogonalize(a["G"], a["ldg"], a["m"], a["n"], a["steps"], None, a["eps"], a["out"],
                                      a["ldo"], a["dtype"], None, 0, None)
    assert call(a) == _lib.ERR_WORKSPACE
    a.update(bad)
    assert call(a) == _lib.ERR_INVALID_ARG


def test_binding_refuses_what_is_not_on_the_gpu():
    x, w = torch.zeros(4, 8), torch.zeros(3, 8)
    for call in (lambda: q.dense_forward(x, w), lambda: q.dense_backward(torch.zeros(4, 3), x, w),
                 lambda: q.xent_forward(x, w, torch.zeros(4, dtype=torch.int64)),
                 lambda: q.xent_grad(x, w, torch.zeros(4, dtype=torch.int64)), lambda: q.orthogonalize(x),
                 lambda: q.orthogonalize(None)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_workspaces_without_alignment_are_no_smaller(dtype):
    for N in (1, 4, 5, 8, 9, 100):
        for Cs, Ct in ((4096, 4096), (4096, 1000), (70, 30), (2047, 3001)):
            for query, more in (("qcnn_dense_forward_workspace_size", ()), ("qcnn_xent_workspace_size", (0,)),
                                ("qcnn_xent_workspace_size", (1,))):
                any_, aligned = (_bytes(query, N, Cs, Ct, dtype, a, *more) for a in (0, 1))
                assert any_ >= aligned
                if dtype == F32:
                    assert any_ == aligned
