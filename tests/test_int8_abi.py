"""Argument checks and workspace queries of dropout and of the 8-bit dense layers, and the plain
forms' generator: host-side, no kernel is launched."""
import ctypes

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from paper_1512_06473_gb300 import _lib, finetune, int8
from test_finetune_devices import _on

lib = _lib.load()
F32, BF16 = _lib.F32, _lib.BF16
P = 256  # a pointer that is aligned and never followed


def test_known_answers_of_the_generator():
    # the published vectors of Philox-4x32-10
    assert plain.philox(0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 2 ** 64 - 1
    assert plain.philox(ones, ones, ones) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert plain.philox(0x85a308d3243f6a88, 0x0370734413198a2e, 0x299f31d0a4093822) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]
    got = plain.words(10, 2 ** 40 + 7, 2 ** 63 + 5, first=2 ** 36)
    assert got.tolist() == sum((plain.philox(2 ** 34 + i, 2 ** 40 + 7, 2 ** 63 + 5) for i in range(3)), [])[:10]


def _dropout(back=False, x=P, ldx=32, N=16, C=32, p=0.5, seed=1, offset=0, add=None, r=None, ldr=0, y=P, ldy=32,
             dtype=F32):
    if back:
        return lib.qcnn_dropout_backward(x, ldx, N, C, p, seed, offset, add, y, ldy, dtype, None)
    return lib.qcnn_dropout_forward(x, ldx, N, C, p, seed, offset, add, r, ldr, y, ldy, dtype, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad", [
    dict(x=None), dict(ldx=31), dict(N=-1), dict(C=0), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")),
    dict(add=P + 4), dict(y=None), dict(ldy=31), dict(dtype=2), dict(x=P + 2), dict(y=P + 2),
    dict(x=P + 1, dtype=BF16)])
def test_dropout_refuses(back, bad):
    assert _dropout(back, **bad) == _lib.ERR_INVALID_ARG


def test_dropout_refuses_a_bad_residual():
    assert _dropout(r=P, ldr=31) == _lib.ERR_INVALID_ARG
    assert _dropout(r=P + 2, ldr=32) == _lib.ERR_INVALID_ARG


def _quantize(x=P, ldx=32, N=16, C=32, codes=P, ldc=32, scale=P, dtype=F32):
    return lib.qcnn_int8_quantize(x, ldx, N, C, codes, ldc, scale, dtype, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(ldx=31), dict(N=-1), dict(C=0), dict(codes=None), dict(ldc=31), dict(scale=None),
    dict(scale=P + 2), dict(dtype=2), dict(x=P + 2), dict(x=P + 1, dtype=BF16)])
def test_quantize_refuses(bad):
    assert _quantize(**bad) == _lib.ERR_INVALID_ARG


def _size(N, Cs, Ct, codes, aligned):
    nb = ctypes.c_size_t()
    assert lib.qcnn_int8_dense_workspace_size(N, Cs, Ct, codes, aligned, ctypes.byref(nb)) == _lib.OK
    return nb.value


def _dense(x=P, ldx=64, xs=None, N=16, Cs=64, W=P, ldw=64, ws=P, Ct=32, bias=None, act=0, r=None, ldr=0, y=P, ldy=32,
           dtype=F32, work=P, wsb=0):
    return lib.qcnn_int8_dense_forward(x, ldx, xs, N, Cs, W, ldw, ws, Ct, bias, act, r, ldr, y, ldy, dtype, work,
                                       wsb, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(ldx=63), dict(N=-1), dict(Cs=0), dict(Ct=0), dict(W=None), dict(ldw=63), dict(ws=None),
    dict(ws=P + 2), dict(act=4), dict(act=-1), dict(bias=P + 2), dict(r=P, ldr=31), dict(r=P + 2, ldr=32),
    dict(y=None), dict(ldy=31), dict(y=P + 2), dict(dtype=2), dict(x=P + 2), dict(xs=P + 2),
    dict(Cs=131072, ldx=131072, ldw=131072)])
def test_dense_refuses(bad):
    assert _dense(**bad) == _lib.ERR_INVALID_ARG


def test_dense_wants_its_workspace():
    large = dict(N=300, Cs=2000, Ct=1000, ldx=2000, ldw=2000, ldy=1000)
    need = _size(300, 2000, 1000, 0, 1)
    assert need > 0
    assert _dense(**large, wsb=need - 1) == _lib.ERR_WORKSPACE
    assert _dense(**large, work=None, wsb=need) == _lib.ERR_WORKSPACE
    assert _dense(**large, work=P + 128, wsb=need) == _lib.ERR_WORKSPACE


def test_nothing_to_do_is_done():
    assert _dropout(N=0, x=None, y=None) == _lib.OK
    assert _quantize(N=0, x=None, codes=None, scale=None) == _lib.OK
    assert _dense(N=0, x=None, y=None, work=None) == _lib.OK
    assert _size(0, 64, 32, 0, 0) == 0


def test_workspaces():
    nb = ctypes.c_size_t()
    assert lib.qcnn_int8_dense_workspace_size(1, 1, 1, 0, 0, None) == _lib.ERR_INVALID_ARG
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (1, 131072, 1)):
        assert lib.qcnn_int8_dense_workspace_size(*bad, 0, 0, ctypes.byref(nb)) == _lib.ERR_INVALID_ARG
    # few rows need none
    assert _size(8, 4096, 1000, 0, 0) == 0 and _size(64, 512, 1000, 1, 0) == 0
    for N in (1, 4, 8, 9, 16, 100, 3001):
        for Cs, Ct in ((4096, 4096), (4096, 1000), (70, 30), (2047, 3001), (131071, 5)):
            for codes in (0, 1):
                assert _size(N, Cs, Ct, codes, 0) >= _size(N, Cs, Ct, codes, 1)


# ------------------------------------------------------------------ binding
X, W, Y = (12, 16), (10, 16), (12, 10)
I8 = dict(dtype=torch.int8)
DENSE = [("x", X, {}), ("weight", W, I8), ("wscale", (10,), {}), ("bias", (10,), {}), ("residual", Y, {}),
         ("out", Y, {})]
CALLS = [
    ("dropout_forward", [("x", X, {}), ("residual", X, {}), ("out", X, {})], dict(p=0.5, seed=1)),
    ("dropout_backward", [("dy", X, {}), ("out", X, {})], dict(p=0.5, seed=1)),
    ("int8_quantize", [("x", X, {}), ("out", X, I8)], {}),
    ("int8_dense_forward", DENSE, {}),
    ("int8_dense_forward", [("x", X, I8), ("xscale", (12,), {})] + DENSE[1:], {}),
]


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(finetune, "_device", lambda: 0)
    for module in (finetune, int8):
        monkeypatch.setattr(module, "load", lambda: pytest.fail("the call went on to the library"))


@pytest.mark.parametrize("name,args,more", CALLS)
def test_another_device_is_refused(host, name, args, more):
    for other in [a[0] for a in args]:
        given = {n: _on(int(n == other), *shape, **kw) for n, shape, kw in args}
        with pytest.raises(ValueError, match="device"):
            getattr(q, name)(**given, **more)
    with pytest.raises(ValueError, match="device"):
        getattr(q, name)(**{n: _on(1, *shape, **kw) for n, shape, kw in args}, **more)


@pytest.mark.parametrize("name,args,more", CALLS)
def test_what_is_no_tensor_or_another_type_is_refused(host, name, args, more):
    for bad in [a[0] for a in args]:
        for wrong in ([0.0], torch.zeros(12, 16)):
            given = {n: wrong if n == bad else _on(0, *shape, **kw) for n, shape, kw in args}
            with pytest.raises(TypeError, match=bad):
                getattr(q, name)(**given, **more)
        given = {n: _on(0, *shape, dtype=torch.float64) if n == bad else _on(0, *shape, **kw)
                 for n, shape, kw in args}
        with pytest.raises(TypeError):
            getattr(q, name)(**given, **more)


@pytest.mark.parametrize("name,args,more", CALLS)
def test_another_shape_is_refused(host, name, args, more):
    for bad in [a[0] for a in args][1:]:
        given = {n: _on(0, *(s + 1 for s in shape), **kw) if n == bad else _on(0, *shape, **kw)
                 for n, shape, kw in args}
        with pytest.raises(ValueError, match="shape"):
            getattr(q, name)(**given, **more)


@pytest.mark.parametrize("bad", [dict(p=1.0), dict(p=-0.5), dict(p=float("nan")), dict(seed=-1), dict(seed=1 << 64),
                                 dict(offset=-1), dict(offset=1 << 64)])
@pytest.mark.parametrize("name", ["dropout_forward", "dropout_backward"])
def test_dropout_numbers(host, name, bad):
    with pytest.raises(ValueError):
        getattr(q, name)(_on(0, *X), **{**dict(p=0.5, seed=1), **bad})


@pytest.mark.parametrize("name", ["dropout_forward", "dropout_backward"])
def test_dropout_offset_tensors(host, name):
    with pytest.raises(TypeError, match="offset"):
        getattr(q, name)(_on(0, *X), 0.5, 1, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError, match="offset"):
        getattr(q, name)(_on(0, *X), 0.5, 1, _on(0, 1))
    for shape, at in (((2,), 0), ((1,), 1)):
        with pytest.raises(ValueError, match="offset"):
            getattr(q, name)(_on(0, *X), 0.5, 1, _on(at, *shape, dtype=torch.int64))


def test_dense_types(host):
    x, w, s = _on(0, *X), _on(0, *W, **I8), _on(0, 10)
    with pytest.raises(TypeError, match="dtype"):
        q.int8_dense_forward(x, w, s, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="dtype"):
        q.int8_dense_forward(_on(0, *X, **I8), w, s, xscale=_on(0, 12), dtype=torch.float16)
    with pytest.raises(TypeError, match="x"):
        q.int8_dense_forward(_on(0, *X, **I8), w, s)
    with pytest.raises(ValueError, match="act"):
        q.int8_dense_forward(x, w, s, act="tanh")
