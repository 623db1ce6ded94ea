"""Dropout and the 8-bit layers as they are used together: a training step of the dense layers behind a
quantized conv stack, its gradients against the formulas' in 64 bits, the step as a graph, and the trained
layers in 8 bits."""
import os
import sys

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _no_timeouts, _normal

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _features(N):
    import finetune_fc
    g = _gen(1)
    net = finetune_fc.conv_stack(g)
    return net.forward(torch.randn(N, 8, finetune_fc.SIDE, finetune_fc.SIDE, generator=g, device="cuda")).flatten(1), g


def _step(x, w1, b1, w2, b2, t, seed, offset, p=0.5):
    h, z = q.dense_forward(x, w1, b1, act="relu", pre=True)
    d = q.dropout_forward(h, p, seed, offset)
    loss, _, dd, dw2, db2 = q.xent_grad(d, w2, t, b2)
    dh = q.dropout_backward(dd, p, seed, offset)
    _, dw1, db1 = q.dense_backward(dh, x, w1, z, "relu", need_dx=False)
    return loss, dw1, db1, dw2, db2


def _head(N=150, hidden=96, classes=11):
    x, g = _features(N)
    w1 = _normal(g, hidden, x.shape[1], scale=(2.0 / x.shape[1]) ** 0.5)
    w2 = _normal(g, classes, hidden, scale=0.2)
    b1, b2 = torch.randn(hidden, generator=g, device="cuda") * 0.1, torch.randn(classes, generator=g, device="cuda")
    t = torch.randint(0, classes, (N,), generator=g, device="cuda")
    t[::9] = -100
    return x, w1, b1, w2, b2, t


def test_gradients_of_a_step():
    x, w1, b1, w2, b2, t = _head()
    seed, offset = 99, 7
    got = _step(x, w1, b1, w2, b2, t, seed, offset)
    p = [v.double().requires_grad_() for v in (w1, b1, w2, b2)]
    z = x.double() @ p[0].T + p[1]
    keep = plain.kept(z.shape, 0.5, offset, seed, "cuda")
    h = torch.where(keep, torch.relu(z) * 2, torch.zeros_like(z))
    loss = torch.nn.functional.cross_entropy(h @ p[2].T + p[3], t, ignore_index=-100, reduction="none")
    (loss.sum() / (t >= 0).sum()).backward()
    assert float((got[0].double() - loss.detach()).abs().max()) <= 1e-5
    # fp32 sums of up to 600 terms, four products one after another: some 10 of 2^-20 of a result's norm
    for a, v in zip(got[1:], p):
        assert float((a.double() - v.grad).norm()) <= 1e-5 * float(v.grad.norm())
    # what the step draws is the offset's
    other = _step(x, w1, b1, w2, b2, t, seed, offset + 1)
    assert not torch.equal(other[1], got[1])


def test_a_step_as_a_graph():
    x, w1, b1, w2, b2, t = _head()
    offset = torch.tensor([3], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(x, w1, b1, w2, b2, t, 5, offset)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = _step(x, w1, b1, w2, b2, t, 5, offset)
        offset.add_(1)
    for step in range(3, 6):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, _step(x, w1, b1, w2, b2, t, 5, step)))


@pytest.mark.parametrize("N", [1, 8, 150, 2000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_trained_layers_in_8_bits(dtype, N):
    """The chain of both layers, each against the plain form of its own input."""
    g = _gen(2)
    x = torch.relu(_normal(g, N, 864, dtype=dtype))
    w1, w2 = _normal(g, 1000, 864, dtype=dtype, scale=0.05), _normal(g, 501, 1000, dtype=dtype, scale=0.05)
    b1, b2 = torch.randn(1000, generator=g, device="cuda"), torch.randn(501, generator=g, device="cuda")
    (c1, s1), (c2, s2) = q.int8_quantize(w1), q.int8_quantize(w2)
    h = q.int8_dense_forward(x, c1, s1, b1, act="relu")
    c, s = plain.quantize(x)
    _near(h, *plain.dense(c.cuda(), s.cuda(), c1, s1, b1, "relu"))
    y = q.int8_dense_forward(h, c2, s2, b2)
    c, s = plain.quantize(h)
    _near(y, *plain.dense(c.cuda(), s.cuda(), c2, s2, b2))
    # and near the dense layers: half a step of each operand
    dense = plain_finetune.dense_forward(h, w2, b2)[0]
    half, rounding = 0.5 + 2.0 ** -15, 2.0 ** -8 if dtype == BF16 else 2.0 ** -20
    s = s.cuda().double()
    bound = half * (h.double().abs().sum(1)[:, None] * s2.double() + s[:, None] * w2.double().abs().sum(1)) + \
        half ** 2 * 1000 * s[:, None] * s2.double()
    assert bool(((y.double() - dense).abs() <= bound + rounding * (dense.abs() + bound)).all())
    _no_timeouts()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_example_runs(dtype):
    import finetune_fc
    losses, right = finetune_fc.main(steps=3, dtype=dtype, show=False, dropout=0.5)
    assert len(losses) == 3 and all(v == v and v < float("inf") for v in losses) and len(right) == 3


@pytest.mark.parametrize("N", [5, 9, 300])
def test_rows_beyond_32_bits(N):
    """Rows so far apart that offsets pass 2^31 elements."""
    ld = (2 ** 31 // (N - 1) + 64) // 64 * 64
    Ct = 500 if N == 300 else 24
    g = _gen(3)
    room = torch.empty(ld * (N - 1) + 4096, dtype=BF16, device="cuda")
    x, y, r = (room.as_strided((N, c), (ld, 1), at) for c, at in ((300, 0), (Ct, 512), (Ct, 1024)))
    x.copy_(torch.randn(N, 300, generator=g, device="cuda"))
    r.copy_(torch.randn(N, Ct, generator=g, device="cuda"))
    w, ws = q.int8_quantize(_normal(g, Ct, 300))
    c, s = plain.quantize(x)
    q.int8_dense_forward(x, w, ws, residual=r, out=y)
    _near(y, *plain.dense(c.cuda(), s.cuda(), w, ws, None, "none", r))
    codes = torch.empty(ld * (N - 1) + 1024, dtype=torch.int8, device="cuda").as_strided((N, 300), (ld, 1))
    _, scale = q.int8_quantize(x, out=codes)
    assert torch.equal(codes.cpu(), c) and torch.equal(scale.cpu(), s)
    far = q.int8_dense_forward(codes, w, ws, xscale=scale, dtype=BF16)
    assert torch.equal(far, q.int8_dense_forward(x, w, ws))
    back = q.int8_dense_forward(w[:min(Ct, N)], codes, scale, xscale=ws[:min(Ct, N)].contiguous())
    _near(back, *plain.dense(w[:min(Ct, N)], ws[:min(Ct, N)], codes, scale))
    near = x.contiguous()
    assert torch.equal(q.dropout_forward(x, 0.5, 1, 2, residual=x), q.dropout_forward(near, 0.5, 1, 2, residual=near))
    del room, x, y, r, codes
    torch.cuda.empty_cache()
