"""The fine-tuning operators at the sizes where another kernel, tile or split takes over:
the results stay within the same bounds (tests/plain_finetune.py)."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune as plain
from test_gpu_finetune import BF16, F32, TYPES, _gen, _near, _no_timeouts, _normal, _xent_case, _xent_near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [4, 5, 8, 9])
@pytest.mark.parametrize("Cs,Ct", [(4096, 300), (4096, 4096), (2048, 8200), (4097, 1000)])
def test_dense_around_eight_rows(N, Cs, Ct, dtype):
    """Weights streamed through multiply-adds or the tensor cores, by their size and alignment."""
    g = _gen(21)
    x, w = _normal(g, N, Cs, dtype=dtype), _normal(g, Ct, Cs, dtype=dtype, scale=1 / math.sqrt(Cs))
    b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    y, z = q.dense_forward(x, w, b, act="silu", residual=r, pre=True)
    wy, wz, ey, ez = plain.dense_forward(x, w, b, "silu", r)
    _near(z, wz, ez, "z")
    _near(y, wy, ey, "y")
    _no_timeouts()


@pytest.mark.parametrize("N", [9, 60, 130])
@pytest.mark.parametrize("Cs", [8, 31, 33, 64, 65, 96, 100, 1060])
@pytest.mark.parametrize("Ct,pad,off", [(64, 0, 0), (300, 4, 0), (300, 1, 1), (20001, 0, 0)])
def test_fp32_weights_split_on_their_way(N, Cs, Ct, pad, off):
    """One block of terms to many, one tile to more than there are SMs, 16-byte rows and not; a
    layer's forward reads its weights' rows, dx (of the transposed shape) their columns."""
    g = _gen(22)
    x, w = _normal(g, N, Cs), _normal(g, Ct, Cs, scale=1 / math.sqrt(Cs), pad=pad, off=off)
    want, _, ey, _ = plain.dense_forward(x, w)
    _near(q.dense_forward(x, w), want, ey)
    dy, v = _normal(g, N, Cs), _normal(g, Cs, Ct, scale=1 / math.sqrt(Cs), pad=pad, off=off)
    dx = q.dense_backward(dy, x.new_zeros(N, Ct), v, need_dweight=False, need_dbias=False)[0]
    want, bound = plain.dense_backward(dy, x.new_zeros(N, Ct), v)
    _near(dx, want[0], bound[0])
    _no_timeouts()


@pytest.mark.parametrize("ld", [1, 2, 3, 5, 30, 33, 66, 131, 1062])
@pytest.mark.parametrize("rows", [1, 3, 4, 5, 31, 33, 127, 130, 515])
def test_fp32_rows_off_16_bytes(rows, ld):
    """Weights whose base is on 16 bytes and whose rows are not, read along and across them; what
    lies between the rows (NaN) goes nowhere."""
    g = _gen(26)
    for cols in {ld, max(1, ld - 3)}:
        w = _normal(g, rows, cols, pad=ld - cols)
        if ld > cols:
            w.as_strided((rows - 1, ld - cols), (ld, 1), w.storage_offset() + cols).fill_(math.nan)
        x, dy = _normal(g, 40, cols), _normal(g, 40, rows)
        want, _, ey, _ = plain.dense_forward(x, w)
        _near(q.dense_forward(x, w), want, ey)
        dx = q.dense_backward(dy, x, w, need_dweight=False, need_dbias=False)[0]
        want, bound = plain.dense_backward(dy, x, w)
        _near(dx, want[0], bound[0])
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,Cs,Ct", [(16, 512, 2000), (64, 128, 20000), (300, 64, 9000), (512, 96, 4100),
                                     (1000, 40, 1000), (2050, 24, 3001), (8, 1024, 9001), (5, 2048, 9000),
                                     (320, 72, 999), (1, 300, 40001), (3, 64, 16384), (38, 40, 16390),
                                     (70, 33, 8200), (2, 8, 4096)])
def test_xent_kept_and_not(N, Cs, Ct, dtype):
    """Logits kept for the call or computed again, in products with few and many shares."""
    g, x, w, b, t = _xent_case(N, Cs, Ct, dtype, seed=23)
    t[N // 2] = -100
    b[Ct // 3] = -math.inf
    t[t == Ct // 3] = 0
    _xent_near(q.xent_forward(x, w, t, b), x, w, t, b)
    _xent_near(q.xent_grad(x, w, t, b), x, w, t, b)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("p", [3, 31, 63, 64, 65])
@pytest.mark.parametrize("q_", [66, 129, 1000, 5000])
def test_orthogonalize_around_64(p, q_, dtype):
    """One launch in shared memory or products, rows or columns the smaller side; the same to what
    rounding leaves (the bound of test_gpu_finetune's)."""
    g = _normal(_gen(24), p, q_, dtype=dtype, scale=3.0)
    want = plain.orthogonalize(g)
    unit = 2.0 ** -24 if dtype == F32 else 2.0 ** -17
    sums = (32 + q_ / (64 if dtype == F32 else 16)) * 2.0 ** -23
    limit = 485 * (unit + sums) * 3 + plain.eps_out(dtype) * float(want.norm())
    for got in (q.orthogonalize(g), q.orthogonalize(g.T.contiguous()).T):
        assert float((got.double() - want).norm()) <= limit
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
def test_workspace_of_any_alignment(dtype):
    """A workspace of the size asked for without alignment serves every matrix."""
    lib, code = q.load(), {F32: 0, BF16: 1}[dtype]
    import ctypes
    g = _gen(25)
    for N in (4, 5, 8, 9, 40):
        for Cs, Ct in ((4096, 64), (512, 4096), (131, 90)):
            nb = ctypes.c_size_t()
            assert lib.qcnn_dense_forward_workspace_size(N, Cs, Ct, code, 0, ctypes.byref(nb)) == 0
            fwd = torch.empty(nb.value + 1, dtype=torch.uint8, device="cuda")[:nb.value]
            assert lib.qcnn_xent_workspace_size(N, Cs, Ct, code, 0, 1, ctypes.byref(nb)) == 0
            grad = torch.empty(nb.value + 1, dtype=torch.uint8, device="cuda")[:nb.value]
            t = torch.randint(0, Ct, (N,), generator=g, device="cuda")
            for pad, off in ((0, 0), (8, 0), (1, 1)):
                x = _normal(g, N, Cs, dtype=dtype, pad=pad, off=off)
                w = _normal(g, Ct, Cs, dtype=dtype, pad=pad, off=off)
                want, _, ey, _ = plain.dense_forward(x, w)
                _near(q.dense_forward(x, w, workspace=fwd), want, ey)
                w = w * (1 / math.sqrt(Cs))
                _xent_near(q.xent_grad(x, w, t, workspace=grad), x, w, t, None)
