"""Dropout on the GPU against its plain 64-bit form: the elements that are kept exactly, the values
within bounds derived in tests/plain_int8.py."""
import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _normal

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]
SEED = 0x9876543210FEDCBA


def _check(x, p, seed, offset, y, r=None):
    want, bound = plain.dropout(x, p, offset, seed, r)
    _near(y, want, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 3), (1, 4), (3, 1), (5, 7), (2, 4096), (128, 64), (33, 1000), (7, 1001),
                                   (100, 4099), (1, 70001), (513, 9)])
def test_forward_and_backward(shape, dtype):
    g = _gen(1)
    x, r = _normal(g, *shape, dtype=dtype), _normal(g, *shape, dtype=dtype)
    for p, offset in ((0.5, 0), (0.1, (1 << 40) + 3)):
        _check(x, p, SEED, offset, q.dropout_forward(x, p, SEED, offset))
        y = q.dropout_forward(x, p, SEED, offset, residual=r)
        _check(x, p, SEED, offset, y, r)
        _check(x, p, SEED, offset, q.dropout_backward(x, p, SEED, offset))
        # on the memory of what is read, element by element
        for mine in (0, 1):
            a, b = x.clone(), r.clone()
            assert torch.equal(q.dropout_forward(a, p, SEED, offset, residual=b, out=(a, b)[mine]), y)
        a = x.clone()
        assert torch.equal(q.dropout_backward(a, p, SEED, offset, out=a), q.dropout_backward(x, p, SEED, offset))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off", [(0, 1), (1, 0), (3, 2), (4, 0), (8, 0), (8, 4), (16, 8)])
@pytest.mark.parametrize("cols", [16, 37, 1024])
def test_strides_and_alignment(cols, pad, off, dtype):
    g = _gen(2)
    x, r = _normal(g, 19, cols, dtype=dtype, pad=pad, off=off), _normal(g, 19, cols, dtype=dtype, pad=pad)
    room = torch.full((19, cols + pad), 7.0, device="cuda", dtype=dtype)
    q.dropout_forward(x, 0.25, SEED, 5, residual=r, out=room[:, :cols])
    _check(x, 0.25, SEED, 5, room[:, :cols], r)
    assert bool((room[:, cols:] == 7).all())  # nothing between the rows is written
    assert torch.equal(q.dropout_backward(x, 0.25, SEED, 5), q.dropout_backward(x.contiguous(), 0.25, SEED, 5))


@pytest.mark.parametrize("dtype", TYPES)
def test_probabilities(dtype):
    x = torch.ones(64, 4096, device="cuda", dtype=dtype)
    assert torch.equal(q.dropout_forward(x, 0.0, 3), x)
    for p in (1e-3, 0.3, 0.999):
        y = q.dropout_forward(x, p, 3)
        _check(x, p, 3, 0, y)
        dropped = float((y == 0).double().mean())
        assert abs(dropped - p) < 6 * (p * (1 - p) / x.numel()) ** 0.5
    assert float((q.dropout_forward(x, 1 - 2.0 ** -40, 3) != 0).sum()) <= 1


def test_offsets_and_seeds_draw_other_words():
    x = torch.ones(32, 4096, device="cuda")
    base = q.dropout_forward(x, 0.5, 1, 0) == 0
    for seed, offset in ((2, 0), (1 << 32 | 1, 0), (1, 1), (1, 1 << 32)):
        same = float((base == (q.dropout_forward(x, 0.5, seed, offset) == 0)).double().mean())
        assert abs(same - 0.5) < 0.02


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_dropped_is_zero_whatever_it_holds(dtype):
    g = _gen(3)
    x = _normal(g, 40, 129, dtype=dtype)
    x[::2, ::3] = float("nan")
    x[1::2, ::3] = float("inf")
    x[1::2, 1::3] = torch.finfo(dtype).max
    for y in (q.dropout_forward(x, 0.5, SEED, 1), q.dropout_backward(x, 0.5, SEED, 1)):
        keep = plain.kept(x.shape, 0.5, 1, SEED, "cuda")
        assert bool((y[~keep] == 0).all())
        assert torch.equal(torch.isnan(y), keep & torch.isnan(x))
        assert torch.equal(torch.isinf(y), keep & (torch.isinf(x) | (x == torch.finfo(dtype).max)))
    r = torch.full_like(x, float("nan"))
    assert bool(torch.isnan(q.dropout_forward(x, 0.5, SEED, 1, residual=r)).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_against_differences(dtype):
    # y is linear in x: (y(x + h) - y(x)) / h is the gradient, within two roundings of y
    g = _gen(4)
    x, dy = _normal(g, 6, 50, dtype=dtype), _normal(g, 6, 50, dtype=dtype)
    dx = q.dropout_backward(dy, 0.25, SEED, 9).double()
    h = 0.5
    up, y = (q.dropout_forward(v, 0.25, SEED, 9).double() for v in ((x.double() + h).to(dtype), x))
    moved = (x.double() + h).to(dtype).double() - x.double()
    slack = plain.kept(x.shape, 0.25, 9, SEED, "cuda") * 2 * 2.0 ** -8 * (up.abs() + y.abs() + dy.double().abs() * 2)
    if dtype == F32:
        slack = slack * 2.0 ** -14
    assert bool(((up - y) * dy.double() - dx * moved).abs().le(slack * (dy.double().abs() + 1)).all())


def test_offset_in_device_memory_and_in_a_graph():
    g = _gen(5)
    x = _normal(g, 64, 1000)
    offset = torch.tensor([17], device="cuda")
    assert torch.equal(q.dropout_forward(x, 0.5, SEED, offset), q.dropout_forward(x, 0.5, SEED, 17))
    out, back = torch.empty_like(x), torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        offset.add_(1)
        q.dropout_forward(x, 0.5, SEED, offset, out=out)
        q.dropout_backward(x, 0.5, SEED, offset, out=back)
    offset.fill_((1 << 45) - 1)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, q.dropout_forward(x, 0.5, SEED, (1 << 45) + step))
        assert torch.equal(back, out)


@pytest.mark.parametrize("dtype", TYPES)
def test_other_streams(dtype):
    g = _gen(6)
    x = _normal(g, 200, 1001, dtype=dtype)
    want = q.dropout_forward(x, 0.5, 1, 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = q.dropout_forward(x, 0.5, 1, 2, stream=s)
    raw = q.dropout_backward(x, 0.5, 1, 2, stream=s.cuda_stream)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want) and torch.equal(raw, want)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    x = torch.empty(0, 5, device="cuda", dtype=dtype)
    assert q.dropout_forward(x, 0.5, 1).shape == (0, 5)
    assert q.dropout_backward(x, 0.5, 1).shape == (0, 5)


def test_elements_beyond_32_bits():
    rows, cols = 70003, 65536  # 4.6 10^9 elements of bf16
    x = torch.ones(rows, cols, device="cuda", dtype=BF16)
    q.dropout_forward(x, 0.5, SEED, 3, out=x)
    for row in (0, 32767, 32768, 65535, 65536, rows - 1):
        keep = plain.words(cols, 3, SEED, first=row * cols, device="cuda") >= 1 << 31
        assert torch.equal(x[row], keep.to(BF16) * 2)
    wide = x[:, :cols - 2]  # rows apart, off the vectors
    q.dropout_backward(wide, 0.0, SEED, 3, out=wide)
    assert torch.equal(x[rows - 1], (plain.words(cols, 3, SEED, first=(rows - 1) * cols, device="cuda") >= 1 << 31)
                       .to(BF16) * 2)
    del x, wide
    torch.cuda.empty_cache()
