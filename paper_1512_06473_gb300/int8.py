"""Dense layers in 8-bit integers, for fine-tuned layers that are to be small without codebooks:
weights as codes with a scale per output, inputs quantized row by row as they come.

Codes are int8 CUDA tensors whose rows may be any distance apart; those that int8_quantize makes
begin every row on 16 bytes, which the products read as they are.  Tensors, devices, streams and
workspaces are as in the fine-tuning calls (finetune.py).
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import _lib, _made_on, _scratch, _workspace, finetune
from ._lib import load
from .finetune import _DTYPES, _F32, _act, _first, _here, _matrix, _new, _vector

_I8 = torch.int8


def int8_quantize(x: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None):
    """(codes [N, C] int8, scale [N] float32) of the rows of x [N, C]: scale = the row's largest
    magnitude times 1/127, codes the whole numbers nearest to x times 1/scale, each step rounded to
    fp32 (qcnn_int8_quantize).  Of dense weights [Ct, Cs] they are what int8_dense_forward takes."""
    code, dev = _first(x, "x")
    ldx = _matrix(x, "x", x.dtype, dev)
    N, C = x.shape
    if out is None:
        ldo = (C + 15) & ~15
        if ldo == C:
            out = _new(x, (N, C), _I8, stream)
        else:  # (rows on 16 bytes in one step: a slice of whole rows takes 5 us more)
            out = _made_on(stream, x.device,
                           lambda: torch.empty_strided((N, C), (ldo, 1), dtype=_I8, device=x.device))
    else:
        ldo = _matrix(out, "out", _I8, dev, N, C)
    scale = _new(x, (N,), _F32, stream)
    st = load().qcnn_int8_quantize(x.data_ptr(), ldx, N, C, out.data_ptr(), ldo, scale.data_ptr(), code,
                                   _here(stream, dev))
    if st:
        _lib.check(st, "qcnn_int8_quantize")
    return out, scale


def int8_route(N: int, Cs: int, Ct: int):
    """How int8_dense_forward goes about these sizes (qcnn_int8_route_info): a dict with "few" (rows
    summed without the tensor cores), "rows" of x and "ctas" per tile, and "shares" of its terms
    (all 0 where few)."""
    info = (ctypes.c_int * 4)()
    _lib.check(load().qcnn_int8_route_info(N, Cs, Ct, info), "qcnn_int8_route_info")
    d = dict(zip(("few", "rows", "ctas", "shares"), list(info)))
    d["few"] = bool(d["few"])
    return d


def int8_dense_forward(x: torch.Tensor, weight: torch.Tensor, wscale: torch.Tensor,
                       bias: Optional[torch.Tensor] = None, act: str = "none",
                       residual: Optional[torch.Tensor] = None, xscale: Optional[torch.Tensor] = None,
                       dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, workspace=None,
                       stream=None):
    """y = act(z) + residual with z = xscale wscale (codes of x) weight^T + bias: dense_forward with
    weights [Ct, Cs] int8 and their scales wscale [Ct] from int8_quantize.  x [N, Cs] float32 or
    bfloat16, whose rows the call quantizes; or, with xscale [N], int8 codes.  y and residual [N, Ct]
    are of ``dtype``: x's type, of codes float32 unless given.  bias, act and ``out`` as in
    dense_forward."""
    codes = xscale is not None
    if codes:
        if not isinstance(x, torch.Tensor) or not x.is_cuda:
            raise TypeError("x must be a CUDA tensor")
        dev = x.get_device()
        if dev != finetune._device():
            raise ValueError(f"x must be on the current device, {finetune._device()}, not on device {dev}")
        dt = _F32 if dtype is None else dtype
        code = _DTYPES.get(dt)
        if code is None:
            raise TypeError(f"dtype must be float32 or bfloat16, got {dt}")
        ldx = _matrix(x, "x", _I8, dev)
    else:
        code, dev = _first(x, "x")
        dt = x.dtype
        if dtype is not None and dtype != dt:
            raise TypeError(f"dtype must be that of x, {dt}, got {dtype}")
        ldx = _matrix(x, "x", dt, dev)
    N, Cs = x.shape
    xs = _vector(xscale, "xscale", _F32, dev, N) if codes else None
    ldw = _matrix(weight, "weight", _I8, dev, None, Cs)
    Ct = weight.shape[0]
    wsc = _vector(wscale, "wscale", _F32, dev, Ct)
    b = None if bias is None else _vector(bias, "bias", _F32, dev, Ct)
    ldr = 0 if residual is None else _matrix(residual, "residual", dt, dev, N, Ct)
    ldy = Ct if out is None else _matrix(out, "out", dt, dev, N, Ct)
    a = _act(act)
    lib = load()
    aligned = not (ldw & 15 or weight.data_ptr() & 15 or (codes and (ldx & 15 or x.data_ptr() & 15)))
    nb = _scratch(lib, "qcnn_int8_dense_workspace_size", N, Cs, Ct, int(codes), int(aligned))
    ws, wsb = _workspace(nb, x.device, workspace, stream) if nb else (None, 0)
    if out is None:
        out = _new(x, (N, Ct), dt, stream)
    st = lib.qcnn_int8_dense_forward(x.data_ptr(), ldx, xs, N, Cs, weight.data_ptr(), ldw, wsc, Ct, b, a,
                                     None if residual is None else residual.data_ptr(), ldr, out.data_ptr(), ldy,
                                     code, ws.data_ptr() if nb else None, wsb, _here(stream, dev))
    if st:
        _lib.check(st, "qcnn_int8_dense_forward")
    return out
