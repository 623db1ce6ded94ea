"""Dropout of matrices large enough for four vectors per thread (from 2^19 vectors of 16 bytes on) and
for counters beyond 32 bits (from 2^34 elements on), in every layout."""
import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _normal

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SEED = 0xFEDCBA9876543210


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counter", [False, True])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("shape", [(3001, 5003), (1100, 4096), (1, 5000001)])
def test_four_vectors_per_thread(shape, pad, counter, dtype):
    g = _gen(1)
    x, r = _normal(g, *shape, dtype=dtype, pad=pad), _normal(g, *shape, dtype=dtype, pad=pad)
    assert x.numel() * x.element_size() >= 16 << 19
    offset = (1 << 33) + 5
    at = torch.tensor([offset], device="cuda") if counter else offset
    for res in (None, r):
        want, bound = plain.dropout(x, 0.3, offset, SEED, res)
        y = q.dropout_forward(x, 0.3, SEED, at, residual=res)
        _near(y, want, bound)
        room = torch.full((shape[0], shape[1] + pad), 7.0, device="cuda", dtype=dtype)
        q.dropout_forward(x, 0.3, SEED, at, residual=res, out=room[:, :shape[1]])
        assert torch.equal(room[:, :shape[1]], y)
        assert bool((room[:, shape[1]:] == 7).all())
        if res is None:
            assert torch.equal(q.dropout_backward(x, 0.3, SEED, at), y)
        # on the memory of what is read
        for mine in ((0,) if res is None else (0, 1)):
            a, b = x.clone(), None if res is None else r.clone()
            assert torch.equal(q.dropout_forward(a, 0.3, SEED, at, residual=b, out=(a, b)[mine]), y)


def _rows_of(x, rows, seed, offset, scale):
    """Rows against the words of their elements; p = 1/2."""
    cols = x.shape[1]
    for row in rows:
        n = row * cols
        first = n // 4 * 4
        w = plain.words(cols + n - first, offset, seed, first=first, device="cuda")[n - first:]
        assert torch.equal(x[row], (w >= 1 << 31).to(x.dtype) * scale), row


def test_rows_apart_beyond_32_bits():
    rows, cols = 70003, 65536  # 4.6 10^9 elements of bf16
    x = torch.ones(rows, cols, device="cuda", dtype=BF16)
    for width in (cols - 2, cols - 8):  # off the vectors, and whole vectors
        x.fill_(1.0)
        view = x[:, :width]
        q.dropout_backward(view, 0.5, SEED, 4, out=view)
        _rows_of(view, (0, 1, 32767, 32768, 65535, 65536, 65540, 65541, rows - 1), SEED, 4, 2.0)
        assert bool((x[:, width:] == 1).all())
    del x, view
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_counters_beyond_32_bits(dtype):
    """34 and 69 GB, in place: rows on 16 bytes (fp32: vectors beyond 32 bits too), then no gaps."""
    rows, cols = 262150, 65536
    room = torch.ones(rows, cols + 8, device="cuda", dtype=dtype)
    view = room[:, :cols]
    some = (0, 1, 65535, 65536, 131072, 262143, 262144, 262145, rows - 1)  # 2^34 elements: from row 262144 on
    q.dropout_forward(view, 0.5, SEED, 6, out=view)
    _rows_of(view, some, SEED, 6, 2.0)
    assert bool((room[some, cols:] == 1).all())
    room.fill_(1.0)
    flat = room.view(-1)[:rows * cols].view(rows, cols)
    q.dropout_forward(flat, 0.5, SEED, 7, out=flat)
    _rows_of(flat, some, SEED, 7, 2.0)
    del room, view, flat
    torch.cuda.empty_cache()
