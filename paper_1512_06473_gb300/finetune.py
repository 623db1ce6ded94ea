"""The operators that fine-tune the dense layers of a network whose conv layers are
quantized (the paper's Sec. 4.2.3), before those are quantized as well: a dense layer
with its epilogue and its backward pass, dropout whose mask is never stored, softmax cross
entropy with its gradient, and the orthogonalised update of a weight matrix.

Matrices are CUDA tensors of one type, float32 or bfloat16, whose rows may be any
distance apart (the columns of a row are neighbours); bias, losses and their gradients
are float32.  Weights are [Ct, Cs], as pq_quantize_fc takes them.  All tensors of a call are on
the current device; an ``out`` overlaps no input but where that is said.  The gradients are calls
of their own: no call is recorded for autograd.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _device, _empty, _lib, _raw_stream, _scratch, _stream, _workspace
from ._lib import load

_DTYPES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}
_F32, _I64 = torch.float32, torch.int64


def _first(t, name):
    """The type code and the device of a call's first matrix; the others' devices are held to it."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    dev = t.get_device()
    if dev != _device():
        raise ValueError(f"{name} must be on the current device, {_device()}, not on device {dev}")
    return code, dev


def _refuse(t, name, dtype, dev, want):
    """What is wrong with a tensor that should be a CUDA tensor of this type, device and shape."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on device {dev}, as the others, not on device {t.get_device()}")
    raise ValueError(f"{name} must be of shape {want}, columns next to each other and rows apart, "
                     f"got shape {tuple(t.shape)} with strides {t.stride()}")


# (a call's host time is its own with small sizes: 0.7 us per matrix, 1.6 per new tensor)
def _matrix(t, name, dtype, dev, rows=None, cols=None):
    """The distance between the rows of a matrix [rows, cols] (None: any)."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.get_device() == dev:
        shape = t.shape
        if len(shape) == 2:
            r, c = shape
            if (rows is None or r == rows) and (cols is None or c == cols):
                ld, unit = t.stride()
                if unit == 1 or c <= 1:
                    if ld >= c:
                        return ld
                    if r <= 1:
                        return c
    _refuse(t, name, dtype, dev, tuple("any" if v is None else v for v in (rows, cols)))


def _vector(t, name, dtype, dev, n):
    # (attributes by themselves: a comparison of shapes makes a tuple, 0.2 us)
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.get_device() == dev and t.dim() == 1 and \
            t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, name, dtype, dev, (n,))


def _here(stream, dev):
    """_stream's handle, dev being the current device."""
    return _raw_stream(dev) if stream is None else _stream(stream)


def _aligned(code, x, ldx, w, ldw):
    """Whether TMA can read both as they are (qcnn.h: aligned)."""
    return 1 if code == _lib.F32 else \
        int(not ((ldx | ldw) & 7 or (x.data_ptr() | w.data_ptr()) & 15))


def _act(act):
    code = _lib.ACT.get(act)
    if code is None:
        raise ValueError(f"act must be one of {sorted(_lib.ACT)}, got {act!r}")
    return code


def _new(like, shape, dtype, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    return _empty(shape, dtype, like.device, stream)


def dense_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  act: str = "none", residual: Optional[torch.Tensor] = None, pre: bool = False,
                  out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """y = act(z) + residual with z = x weight^T + bias, in one product with its
    epilogue.  x [N, Cs], weight [Ct, Cs], bias [Ct] float32, residual [N, Ct]; act is
    "none", "relu", "gelu" (by erf) or "silu"; ``out`` may be residual.  pre=True returns (y, z): z is what
    dense_backward needs."""
    code, dev = _first(x, "x")
    dt = x.dtype
    ldx = _matrix(x, "x", dt, dev)
    N, Cs = x.shape
    ldw = _matrix(weight, "weight", dt, dev, None, Cs)
    Ct = weight.shape[0]
    b = None if bias is None else _vector(bias, "bias", _F32, dev, Ct)
    ldr = 0 if residual is None else _matrix(residual, "residual", dt, dev, N, Ct)
    ldy = Ct if out is None else _matrix(out, "out", dt, dev, N, Ct)
    a = _act(act)
    lib = load()
    nb = _scratch(lib, "qcnn_dense_forward_workspace_size", N, Cs, Ct, code,
                  _aligned(code, x, ldx, weight, ldw))
    ws, wsb = _workspace(nb, x.device, workspace, stream) if nb else (None, 0)
    if out is None:
        out = _new(x, (N, Ct), dt, stream)
    z = _new(x, (N, Ct), dt, stream) if pre else None
    st = lib.qcnn_dense_forward(x.data_ptr(), ldx, N, Cs, weight.data_ptr(), ldw, Ct, b, a,
                                None if residual is None else residual.data_ptr(), ldr,
                                out.data_ptr(), ldy, z.data_ptr() if pre else None, Ct, code,
                                ws.data_ptr() if nb else None, wsb, _stream(stream))
    if st:
        _lib.check(st, "qcnn_dense_forward")
    return (out, z) if pre else out


def dense_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                   pre: Optional[torch.Tensor] = None, act: str = "none", need_dx: bool = True,
                   need_dweight: bool = True, need_dbias: bool = True, workspace=None, stream=None):
    """The gradients (dx, dweight, dbias) of dense_forward for the gradient dy [N, Ct] of
    y, with pre = z (not needed for act "none"; for a ReLU without residual y will do).
    What is not needed is None.  The residual's gradient is dy itself."""
    code, dev = _first(dy, "dy")
    dt = dy.dtype
    lddy = _matrix(dy, "dy", dt, dev)
    N, Ct = dy.shape
    ldx = _matrix(x, "x", dt, dev, N)
    Cs = x.shape[1]
    ldw = _matrix(weight, "weight", dt, dev, Ct, Cs)
    a = _act(act)
    if a and pre is None:
        raise ValueError(f"pre is required with act {act!r}")
    ldp = 0 if pre is None else _matrix(pre, "pre", dt, dev, N, Ct)
    lib = load()
    nb = _scratch(lib, "qcnn_dense_backward_workspace_size", N, Cs, Ct, code,
                  _aligned(code, x, ldx, weight, ldw))
    ws, wsb = _workspace(nb, dy.device, workspace, stream) if nb else (None, 0)
    dx = _new(dy, (N, Cs), dt, stream) if need_dx else None
    dw = _new(dy, (Ct, Cs), dt, stream) if need_dweight else None
    db = _new(dy, (Ct,), _F32, stream) if need_dbias else None
    st = lib.qcnn_dense_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, weight.data_ptr(), ldw,
                                 None if pre is None else pre.data_ptr(), ldp,
                                 N, Cs, Ct, a, dx.data_ptr() if need_dx else None, Cs,
                                 dw.data_ptr() if need_dweight else None, Cs,
                                 db.data_ptr() if need_dbias else None, code,
                                 ws.data_ptr() if nb else None, wsb, _stream(stream))
    if st:
        _lib.check(st, "qcnn_dense_backward")
    return dx, dw, db


def _xent_args(x, weight, targets, bias):
    code, dev = _first(x, "x")
    ldx = _matrix(x, "x", x.dtype, dev)
    N, Cs = x.shape
    ldw = _matrix(weight, "weight", x.dtype, dev, None, Cs)
    Ct = weight.shape[0]
    t = _vector(targets, "targets", _I64, dev, N)
    b = None if bias is None else _vector(bias, "bias", _F32, dev, Ct)
    return code, dev, ldx, ldw, N, Cs, Ct, t, b


def xent_route(N: int, Cs: int, Ct: int, dtype=torch.float32, grad: bool = True):
    """How xent_grad (or, grad False, xent_forward) goes about these sizes
    (qcnn_xent_route_info): a dict with "kept" (the logits), classes of a "piece" and of the
    "last" one, "pieces", and "shares" of a tile's classes in the last piece's dx, of
    "share_classes" each (both 0 without grad)."""
    if dtype not in _DTYPES:
        raise TypeError(f"dtype must be float32 or bfloat16, got {dtype}")
    info = (ctypes.c_int * 6)()
    _lib.check(load().qcnn_xent_route_info(N, Cs, Ct, _DTYPES[dtype], int(grad), info),
               "qcnn_xent_route_info")
    d = dict(zip(("kept", "piece", "last", "pieces", "shares", "share_classes"), list(info)))
    d["kept"] = bool(d["kept"])
    return d


def xent_forward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                 bias: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """Softmax cross entropy of the logits x weight^T + bias: (loss [N], lse [N]), float32,
    with lse the log of the sum of exp of a row's logits and loss = lse - logit of the
    row's target.  x [N, Cs], weight [Ct, Cs], targets [N] int64, bias [Ct] float32
    (-inf takes a class out).  A row with a negative target has loss 0.  The logits are
    not kept where they would be large."""
    code, _, ldx, ldw, N, Cs, Ct, t, b = _xent_args(x, weight, targets, bias)
    lib = load()
    nb = _scratch(lib, "qcnn_xent_workspace_size", N, Cs, Ct, code,
                  _aligned(code, x, ldx, weight, ldw), 0)
    ws, wsb = _workspace(nb, x.device, workspace, stream) if nb else (None, 0)
    loss, lse = _new(x, (N,), _F32, stream), _new(x, (N,), _F32, stream)
    st = lib.qcnn_xent_forward(x.data_ptr(), ldx, N, Cs, weight.data_ptr(), ldw, Ct, b, t,
                               loss.data_ptr(), lse.data_ptr(), code, ws.data_ptr() if nb else None,
                               wsb, _stream(stream))
    if st:
        _lib.check(st, "qcnn_xent_forward")
    return loss, lse


def xent_grad(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
              bias: Optional[torch.Tensor] = None, dloss: Optional[torch.Tensor] = None,
              workspace=None, stream=None):
    """xent_forward with the gradients of sum(dloss * loss), or (dloss None) of the mean
    of the losses over the rows with a target: (loss, lse, dx [N, Cs], dweight [Ct, Cs],
    dbias [Ct] float32).  Rows with a negative target have gradient 0."""
    code, dev, ldx, ldw, N, Cs, Ct, t, b = _xent_args(x, weight, targets, bias)
    d = None if dloss is None else _vector(dloss, "dloss", _F32, dev, N)
    lib = load()
    nb = _scratch(lib, "qcnn_xent_workspace_size", N, Cs, Ct, code,
                  _aligned(code, x, ldx, weight, ldw), 1)
    ws, wsb = _workspace(nb, x.device, workspace, stream) if nb else (None, 0)
    loss, lse = _new(x, (N,), _F32, stream), _new(x, (N,), _F32, stream)
    dx, dw = _new(x, (N, Cs), x.dtype, stream), _new(x, (Ct, Cs), x.dtype, stream)
    db = _new(x, (Ct,), _F32, stream)
    st = lib.qcnn_xent_grad(x.data_ptr(), ldx, N, Cs, weight.data_ptr(), ldw, Ct, b, t, d,
                            loss.data_ptr(), lse.data_ptr(), dx.data_ptr(), Cs, dw.data_ptr(), Cs,
                            db.data_ptr(), code, ws.data_ptr() if nb else None, wsb, _stream(stream))
    if st:
        _lib.check(st, "qcnn_xent_grad")
    return loss, lse, dx, dw, db


def orthogonalize(g: torch.Tensor, steps: int = 5, coeffs: Optional[Sequence[float]] = None,
                  eps: float = 1e-7, out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """The update g [m, n] with its singular values brought near 1, by ``steps``
    Newton-Schulz steps X <- a X + (b A + c A A) X, A = X X^T, from X = g / (||g||_F +
    eps); coeffs (a, b, c), by default those of the Muon optimiser.  ``out`` may be g."""
    code, dev = _first(g, "g")
    ldg = _matrix(g, "g", g.dtype, dev)
    m, n = g.shape
    if out is None:
        out, ldo = _new(g, (m, n), g.dtype, stream), n
    else:
        ldo = _matrix(out, "out", g.dtype, dev, m, n)
    k = None
    if coeffs is not None:
        if len(coeffs) != 3:
            raise ValueError("coeffs must be three numbers")
        k = (ctypes.c_float * 3)(*coeffs)
    lib = load()
    nb = _scratch(lib, "qcnn_orthogonalize_workspace_size", m, n, code)
    ws, wsb = _workspace(nb, g.device, workspace, stream)
    _lib.check(lib.qcnn_orthogonalize(g.data_ptr(), ldg, m, n, int(steps), k, float(eps),
                                      out.data_ptr(), ldo, code, ws.data_ptr(), wsb,
                                      _stream(stream)), "qcnn_orthogonalize")
    return out


def _dropout(name, x, x_name, p, seed, offset, residual, out, stream):
    code, dev = _first(x, x_name)
    dt = x.dtype
    ldx = _matrix(x, x_name, dt, dev)
    N, C = x.shape
    if not 0.0 <= p < 1.0:
        raise ValueError(f"p must be at least 0 and below 1, got {p}")
    if not 0 <= seed < 1 << 64:
        raise ValueError(f"seed must be a number of 64 bits, got {seed}")
    add = None
    if isinstance(offset, torch.Tensor):
        if offset.dtype is not _I64 or not offset.is_cuda or offset.get_device() != dev or offset.numel() != 1:
            _refuse(offset, "offset", _I64, dev, (1,))
        add, offset = offset.data_ptr(), 0
    elif not 0 <= offset < 1 << 64:
        raise ValueError(f"offset must be a number of 64 bits, got {offset}")
    ldr = 0 if residual is None else _matrix(residual, "residual", dt, dev, N, C)
    if out is not None:
        ldo = _matrix(out, "out", dt, dev, N, C)
    else:
        ldo = C
        out = torch.empty_like(x) if stream is None and ldx == C and x.is_contiguous() else _new(x, (N, C), dt, stream)
    lib = load()
    if name == "qcnn_dropout_forward":
        st = lib.qcnn_dropout_forward(x.data_ptr(), ldx, N, C, p, seed, offset, add,
                                      None if residual is None else residual.data_ptr(), ldr, out.data_ptr(), ldo,
                                      code, _here(stream, dev))
    else:
        st = lib.qcnn_dropout_backward(x.data_ptr(), ldx, N, C, p, seed, offset, add, out.data_ptr(), ldo, code,
                                       _here(stream, dev))
    if st:
        _lib.check(st, name)
    return out


def dropout_forward(x: torch.Tensor, p: float, seed: int, offset=0, residual: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None, stream=None):
    """y = x / (1 - p) where an element is kept, else 0; plus residual.  x, residual [N, C]; 0 <= p < 1;
    ``out`` may be x or residual.  What is kept follows from seed, offset (64 bits each) and an
    element's place (Philox-4x32, qcnn.h), so that nothing is stored: dropout_backward draws it
    again.  Give each call of a step an offset of its own, and the backward call the same; or a CUDA
    int64 tensor of one element, read as the kernel runs, which a captured graph's owner
    can change between replays."""
    return _dropout("qcnn_dropout_forward", x, "x", p, seed, offset, residual, out, stream)


def dropout_backward(dy: torch.Tensor, p: float, seed: int, offset=0, out: Optional[torch.Tensor] = None,
                     stream=None):
    """The gradient of x for the gradient dy [N, C] of dropout_forward's y, with the same p, seed and
    offset.  ``out`` may be dy.  The residual's gradient is dy itself."""
    return _dropout("qcnn_dropout_backward", dy, "dy", p, seed, offset, None, out, stream)
