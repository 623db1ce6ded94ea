"""The operators that fine-tune the dense layers of a network whose conv layers are
quantized (the paper's Sec. 4.2.3), before those are quantized as well: a dense layer
with its epilogue and its backward pass, softmax cross entropy with its gradient, and
the orthogonalised update of a weight matrix.

Matrices are CUDA tensors of one type, float32 or bfloat16, whose rows may be any
distance apart (the columns of a row are neighbours); bias, losses and their gradients
are float32.  Weights are [Ct, Cs], as pq_quantize_fc takes them.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _empty, _lib, _ptr, _scratch, _stream, _workspace
from ._lib import load

_DTYPES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}


def _dtype(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return code


def _matrix(t, name, dtype, rows=None, cols=None):
    """The distance between the rows of a matrix [rows, cols] (None: any)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or \
            (cols is not None and t.shape[1] != cols):
        want = tuple("any" if v is None else v for v in (rows, cols))
        raise ValueError(f"{name} must be of shape {want}, got {tuple(t.shape)}")
    r, c = t.shape
    ld, unit = t.stride()
    if c > 1 and unit != 1:
        raise ValueError(f"the columns of {name} must be neighbours, got strides {t.stride()}")
    if r <= 1:
        return max(ld, c)
    if ld < c:
        raise ValueError(f"the rows of {name} overlap: strides {t.stride()}")
    return ld


def _vector(t, name, dtype, n):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be contiguous of {n} elements, got shape {tuple(t.shape)}")


def _aligned(code, *mats):
    """Whether TMA can read these (tensor, row distance) as they are (qcnn.h: aligned)."""
    if code == _lib.F32:
        return 1
    return int(all(t is None or (t.data_ptr() % 16 == 0 and ld % 8 == 0) for t, ld in mats))


def _act(act):
    code = _lib.ACT.get(act)
    if code is None:
        raise ValueError(f"act must be one of {sorted(_lib.ACT)}, got {act!r}")
    return code


def dense_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  act: str = "none", residual: Optional[torch.Tensor] = None, pre: bool = False,
                  out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """y = act(z) + residual with z = x weight^T + bias, in one product with its
    epilogue.  x [N, Cs], weight [Ct, Cs], bias [Ct] float32, residual [N, Ct]; act is
    "none", "relu", "gelu" (by erf) or "silu".  pre=True returns (y, z): z is what
    dense_backward needs."""
    code = _dtype(x, "x")
    dt = x.dtype
    ldx = _matrix(x, "x", dt)
    N, Cs = x.shape
    ldw = _matrix(weight, "weight", dt, None, Cs)
    Ct = weight.shape[0]
    if bias is not None:
        _vector(bias, "bias", torch.float32, Ct)
    ldr = 0 if residual is None else _matrix(residual, "residual", dt, N, Ct)
    a = _act(act)
    lib = load()
    dev = x.device
    nb = _scratch(lib, "qcnn_dense_forward_workspace_size", N, Cs, Ct, code,
                  _aligned(code, (x, ldx), (weight, ldw)))
    ws, wsb = _workspace(nb, dev, workspace, stream)
    if out is None:
        out = _empty((N, Ct), dt, dev, stream)
    ldy = _matrix(out, "out", dt, N, Ct)
    z = _empty((N, Ct), dt, dev, stream) if pre else None
    _lib.check(lib.qcnn_dense_forward(_ptr(x), ldx, N, Cs, _ptr(weight), ldw, Ct, _ptr(bias), a,
                                      _ptr(residual), ldr, _ptr(out), ldy, _ptr(z), Ct, code,
                                      _ptr(ws), wsb, _stream(stream)), "qcnn_dense_forward")
    return (out, z) if pre else out


def dense_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                   pre: Optional[torch.Tensor] = None, act: str = "none", need_dx: bool = True,
                   need_dweight: bool = True, need_dbias: bool = True, workspace=None, stream=None):
    """The gradients (dx, dweight, dbias) of dense_forward for the gradient dy [N, Ct] of
    y, with pre = z (not needed for act "none"; for a ReLU without residual y will do).
    What is not needed is None.  The residual's gradient is dy itself."""
    code = _dtype(dy, "dy")
    dt = dy.dtype
    lddy = _matrix(dy, "dy", dt)
    N, Ct = dy.shape
    ldx = _matrix(x, "x", dt, N)
    Cs = x.shape[1]
    ldw = _matrix(weight, "weight", dt, Ct, Cs)
    a = _act(act)
    if a and pre is None:
        raise ValueError(f"pre is required with act {act!r}")
    ldp = 0 if pre is None else _matrix(pre, "pre", dt, N, Ct)
    lib = load()
    dev = dy.device
    nb = _scratch(lib, "qcnn_dense_backward_workspace_size", N, Cs, Ct, code,
                  _aligned(code, (x, ldx), (weight, ldw)))
    ws, wsb = _workspace(nb, dev, workspace, stream)
    dx = _empty((N, Cs), dt, dev, stream) if need_dx else None
    dw = _empty((Ct, Cs), dt, dev, stream) if need_dweight else None
    db = _empty((Ct,), torch.float32, dev, stream) if need_dbias else None
    _lib.check(lib.qcnn_dense_backward(_ptr(dy), lddy, _ptr(x), ldx, _ptr(weight), ldw, _ptr(pre), ldp,
                                       N, Cs, Ct, a, _ptr(dx), Cs, _ptr(dw), Cs, _ptr(db), code,
                                       _ptr(ws), wsb, _stream(stream)), "qcnn_dense_backward")
    return dx, dw, db


def _xent_args(x, weight, targets, bias):
    code = _dtype(x, "x")
    ldx = _matrix(x, "x", x.dtype)
    N, Cs = x.shape
    ldw = _matrix(weight, "weight", x.dtype, None, Cs)
    Ct = weight.shape[0]
    _vector(targets, "targets", torch.int64, N)
    if bias is not None:
        _vector(bias, "bias", torch.float32, Ct)
    return code, ldx, ldw, N, Cs, Ct


def xent_forward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                 bias: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """Softmax cross entropy of the logits x weight^T + bias: (loss [N], lse [N]), float32,
    with lse the log of the sum of exp of a row's logits and loss = lse - logit of the
    row's target.  x [N, Cs], weight [Ct, Cs], targets [N] int64, bias [Ct] float32
    (-inf takes a class out).  A row with a negative target has loss 0.  The logits are
    not kept where they would be large."""
    code, ldx, ldw, N, Cs, Ct = _xent_args(x, weight, targets, bias)
    lib = load()
    dev = x.device
    nb = _scratch(lib, "qcnn_xent_workspace_size", N, Cs, Ct, code,
                  _aligned(code, (x, ldx), (weight, ldw)), 0)
    ws, wsb = _workspace(nb, dev, workspace, stream)
    loss = _empty((N,), torch.float32, dev, stream)
    lse = _empty((N,), torch.float32, dev, stream)
    _lib.check(lib.qcnn_xent_forward(_ptr(x), ldx, N, Cs, _ptr(weight), ldw, Ct, _ptr(bias),
                                     _ptr(targets), _ptr(loss), _ptr(lse), code, _ptr(ws), wsb,
                                     _stream(stream)), "qcnn_xent_forward")
    return loss, lse


def xent_grad(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
              bias: Optional[torch.Tensor] = None, dloss: Optional[torch.Tensor] = None,
              workspace=None, stream=None):
    """xent_forward with the gradients of sum(dloss * loss), or (dloss None) of the mean
    of the losses over the rows with a target: (loss, lse, dx [N, Cs], dweight [Ct, Cs],
    dbias [Ct] float32).  Rows with a negative target have gradient 0."""
    code, ldx, ldw, N, Cs, Ct = _xent_args(x, weight, targets, bias)
    if dloss is not None:
        _vector(dloss, "dloss", torch.float32, N)
    lib = load()
    dev = x.device
    nb = _scratch(lib, "qcnn_xent_workspace_size", N, Cs, Ct, code,
                  _aligned(code, (x, ldx), (weight, ldw)), 1)
    ws, wsb = _workspace(nb, dev, workspace, stream)
    loss = _empty((N,), torch.float32, dev, stream)
    lse = _empty((N,), torch.float32, dev, stream)
    dx = _empty((N, Cs), x.dtype, dev, stream)
    dw = _empty((Ct, Cs), x.dtype, dev, stream)
    db = _empty((Ct,), torch.float32, dev, stream)
    _lib.check(lib.qcnn_xent_grad(_ptr(x), ldx, N, Cs, _ptr(weight), ldw, Ct, _ptr(bias),
                                  _ptr(targets), _ptr(dloss), _ptr(loss), _ptr(lse), _ptr(dx), Cs,
                                  _ptr(dw), Cs, _ptr(db), code, _ptr(ws), wsb, _stream(stream)),
               "qcnn_xent_grad")
    return loss, lse, dx, dw, db


def orthogonalize(g: torch.Tensor, steps: int = 5, coeffs: Optional[Sequence[float]] = None,
                  eps: float = 1e-7, out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """The update g [m, n] with its singular values brought near 1, by ``steps``
    Newton-Schulz steps X <- a X + (b A + c A A) X, A = X X^T, from X = g / (||g||_F +
    eps); coeffs (a, b, c), by default those of the Muon optimiser.  ``out`` may be g."""
    code = _dtype(g, "g")
    ldg = _matrix(g, "g", g.dtype)
    m, n = g.shape
    if out is None:
        out = _empty((m, n), g.dtype, g.device, stream)
    ldo = _matrix(out, "out", g.dtype, m, n)
    k = None
    if coeffs is not None:
        if len(coeffs) != 3:
            raise ValueError("coeffs must be three numbers")
        k = (ctypes.c_float * 3)(*coeffs)
    lib = load()
    nb = _scratch(lib, "qcnn_orthogonalize_workspace_size", m, n, code)
    ws, wsb = _workspace(nb, g.device, workspace, stream)
    _lib.check(lib.qcnn_orthogonalize(_ptr(g), ldg, m, n, int(steps), k, float(eps), _ptr(out), ldo,
                                      code, _ptr(ws), wsb, _stream(stream)), "qcnn_orthogonalize")
    return out
