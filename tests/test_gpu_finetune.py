"""The fine-tuning operators on the GPU against their plain 64-bit forms, element by
element within bounds derived there (tests/plain_finetune.py)."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_finetune as plain

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, dtype=F32, scale=1.0, pad=0, off=0):
    """A matrix; pad: columns more between rows; off: elements that its first is off 16 bytes."""
    rows, cols = shape
    buf = torch.randn(rows * (cols + pad) + off, generator=g, device="cuda") * scale
    return buf.to(dtype)[off:].view(rows, cols + pad)[:, :cols]


def _near(got, want, bound, name=""):
    """|got - want| <= bound + got's own rounding, everywhere."""
    got64 = got.double()
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), f"{name}: NaN in other places"
    fine = torch.isfinite(want)
    assert torch.equal(got64[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), name
    limit = bound + plain.eps_out(got.dtype) * (want.abs() + bound) + 1e-38
    over = ((got64 - want).abs() / limit)[fine]
    assert over.numel() == 0 or float(over.max()) <= 1.0, f"{name}: {float(over.max()):.2f} of the bound"


def _no_timeouts():
    assert q.device_check() == 0


DENSE = [  # N, Cs, Ct: few rows, one tile, ragged tiles, split sums, several tiles, short sums
    (1, 1, 1), (1, 64, 64), (1, 4096, 1000), (2, 100, 33), (5, 1001, 7), (8, 520, 130), (9, 64, 16),
    (16, 128, 128), (100, 72, 200), (128, 4096, 256), (129, 300, 127), (257, 64, 513), (300, 515, 301),
    (33, 2000, 1), (700, 1024, 640), (2, 9000, 5000), (130, 1, 140), (64, 129, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", DENSE)
def test_dense_forward(shape, dtype):
    N, Cs, Ct = shape
    g = _gen(1)
    x, w = _normal(g, N, Cs, dtype=dtype), _normal(g, Ct, Cs, dtype=dtype, scale=1 / math.sqrt(Cs))
    b = torch.randn(Ct, generator=g, device="cuda")
    y = q.dense_forward(x, w, b)
    want, _, ey, _ = plain.dense_forward(x, w, b)
    _near(y, want, ey)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(3, 70, 90), (150, 200, 144), (140, 2000, 301)])
def test_dense_forward_epilogues(shape, act, dtype):
    N, Cs, Ct = shape
    g = _gen(2)
    x, w = _normal(g, N, Cs, dtype=dtype, scale=2), _normal(g, Ct, Cs, dtype=dtype, scale=1 / math.sqrt(Cs))
    b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    y, z = q.dense_forward(x, w, b, act=act, residual=r, pre=True)
    wy, wz, ey, ez = plain.dense_forward(x, w, b, act, r)
    _near(z, wz, ez, "z")
    _near(y, wy, ey, "y")
    # the residual's memory may be the output's
    out = r.clone()
    assert torch.equal(q.dense_forward(x, w, b, act=act, residual=out, out=out), y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [4, 40, 300])
@pytest.mark.parametrize("pad,off", [(0, 1), (1, 0), (3, 2), (8, 0), (8, 4)])
def test_dense_strides_and_alignment(N, pad, off, dtype):
    """Rows any distance apart, bases on any element; what lies between rows stays."""
    g = _gen(3)
    Cs, Ct = 131, 98
    x, w = _normal(g, N, Cs, dtype=dtype, pad=pad, off=off), _normal(g, Ct, Cs, dtype=dtype, pad=pad, off=off)
    r = _normal(g, N, Ct, dtype=dtype, pad=pad, off=off)
    buf = torch.full((N, Ct + pad + 2), 7.0, dtype=dtype, device="cuda")
    out = buf[:, 1:Ct + 1]
    q.dense_forward(x, w, None, act="gelu", residual=r, out=out)
    want, _, ey, _ = plain.dense_forward(x, w, None, "gelu", r)
    _near(out, want, ey)
    assert bool((buf[:, 0] == 7).all()) and bool((buf[:, Ct + 1:] == 7).all())
    dy, z = r, _normal(g, N, Ct, dtype=dtype, pad=pad, off=off)
    got = q.dense_backward(dy, x, w, z, "silu")
    want, bound = plain.dense_backward(dy, x, w, z, "silu")
    for a, b, e, n in zip(got, want, bound, ("dx", "dw", "db")):
        _near(a, b, e, n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 200, 300), (7, 65, 33), (64, 64, 64), (128, 512, 256),
                                   (129, 300, 1000), (300, 129, 67), (1030, 520, 260), (65, 4000, 2)])
def test_dense_backward(shape, act, dtype):
    N, Cs, Ct = shape
    g = _gen(4)
    x, w = _normal(g, N, Cs, dtype=dtype), _normal(g, Ct, Cs, dtype=dtype, scale=1 / math.sqrt(Cs))
    dy, z = _normal(g, N, Ct, dtype=dtype, scale=1e-3), _normal(g, N, Ct, dtype=dtype, scale=2)
    z = None if act == "none" else z
    got = q.dense_backward(dy, x, w, z, act)
    want, bound = plain.dense_backward(dy, x, w, z, act)
    for a, b, e, n in zip(got, want, bound, ("dx", "dw", "db")):
        _near(a, b, e, n)
    _no_timeouts()
    # each alone is the same
    only = [q.dense_backward(dy, x, w, z, act, *(i == j for j in range(3))) for i in range(3)]
    for i in range(3):
        assert [v is None for v in only[i]] == [i != j for j in range(3)]
        _near(only[i][i], want[i], bound[i])


@pytest.mark.parametrize("dtype", TYPES)
def test_dense_backward_against_differences(dtype):
    """<gradient, direction> is the difference of the value along it, in 64 bits."""
    g = _gen(5)
    N, Cs, Ct = 40, 96, 72
    x, w = _normal(g, N, Cs, dtype=dtype), _normal(g, Ct, Cs, dtype=dtype, scale=0.1)
    b, dy = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    z = (x.double() @ w.double().T + b.double()).to(dtype)
    got = q.dense_backward(dy, x, w, z, "gelu")
    _, bound = plain.dense_backward(dy, x, w, z, "gelu")

    def value(x, w, b):
        return (plain.act(x @ w.T + b, "gelu") * dy.double()).sum()

    # (z rounded to the type moves the slope by up to 1.2 |dz|)
    ez = plain.eps_out(dtype) * 1.2 * z.double().abs() * dy.double().abs()
    more = (ez @ w.double().abs(), ez.T @ x.double().abs(), ez.sum(0))
    base = [x.double(), w.double(), b.double()]
    for i in range(3):
        v = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + h * v, base[i] - h * v
        diff = float((value(*up) - value(*down)) / (2 * h))
        limit = float(((bound[i] + more[i] + plain.eps_out(got[i].dtype) * got[i].double().abs()) * v.abs()).sum())
        assert abs(float((got[i].double() * v).sum()) - diff) <= limit + 1e-6


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    x, w = torch.empty(0, 24, dtype=dtype, device="cuda"), torch.ones(17, 24, dtype=dtype, device="cuda")
    assert q.dense_forward(x, w).shape == (0, 17)
    dx, dw, db = q.dense_backward(torch.empty(0, 17, dtype=dtype, device="cuda"), x, w)
    assert dx.shape == (0, 24) and not dw.any() and not db.any() and dw.shape == (17, 24)
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = q.xent_forward(x, w, t)
    assert loss.shape == lse.shape == (0,)
    loss, lse, dx, dw, db = q.xent_grad(x, w, t)
    assert dx.shape == (0, 24) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_non_finite_values_stay_where_they_enter(dtype):
    g = _gen(6)
    x, w = _normal(g, 40, 200, dtype=dtype), _normal(g, 48, 200, dtype=dtype)
    x[3, 7] = math.nan
    x[20, 199] = math.inf
    w[5, 0] = -math.inf
    y = q.dense_forward(x, w)
    bad = torch.zeros(40, 48, dtype=torch.bool, device="cuda")
    bad[3] = bad[20] = True
    bad[:, 5] = True
    assert torch.equal(~torch.isfinite(y), bad)
    want, _, ey, _ = plain.dense_forward(x, w)
    _near(y[~bad], want[~bad], ey[~bad])
    # NaN goes through the activations, and infinities of bf16 are theirs
    assert torch.isnan(q.dense_forward(x, w, act="relu")[3]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_large_and_small_values(dtype):
    """fp32 pieces hold 24 bits down to 2^-110 and none is lost below 2^-133."""
    g = _gen(7)
    x, w = _normal(g, 33, 96, dtype=dtype), _normal(g, 40, 96, dtype=dtype)
    for a, b in ((1e25, 1e-25), (1e-30, 1e20), (1e15, 1e15)):
        xs, ws = (x.float() * a).to(dtype), (w.float() * b).to(dtype)
        want, _, ey, _ = plain.dense_forward(xs, ws)
        _near(q.dense_forward(xs, ws), want, ey + 2.0 ** -132 * 96 * max(a, b) * 8)


XENT = [  # N, Cs, Ct: few rows, one class, kept logits, pieces (logits of 64 MB and more)
    (1, 40, 1), (1, 512, 1000), (3, 33, 50), (8, 100, 1001), (9, 64, 16), (100, 130, 10), (128, 1024, 1000),
    (257, 40, 2050), (700, 65, 31), (1100, 72, 16001), (600, 40, 30001)]


def _xent_case(N, Cs, Ct, dtype, seed=8):
    g = _gen(seed)
    x, w = _normal(g, N, Cs, dtype=dtype), _normal(g, Ct, Cs, dtype=dtype, scale=2 / math.sqrt(Cs))
    b = torch.randn(Ct, generator=g, device="cuda")
    t = torch.randint(0, Ct, (N,), generator=g, device="cuda")
    return g, x, w, b, t


def _xent_near(got, x, w, t, b, dloss=None):
    want, bound = plain.xent(x, w, t, b, dloss)
    for a, c, e, n in zip(got, want, bound, ("loss", "lse", "dx", "dw", "db")):
        _near(a, c, e, n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", XENT)
def test_xent(shape, dtype):
    N, Cs, Ct = shape
    g, x, w, b, t = _xent_case(N, Cs, Ct, dtype)
    if N > 2:
        t[1] = -100
        t[N - 1] = -1
    _xent_near(q.xent_forward(x, w, t, b), x, w, t, b)
    _xent_near(q.xent_grad(x, w, t, b), x, w, t, b)
    _xent_near(q.xent_grad(x, w, t), x, w, t, None)
    dloss = torch.randn(N, generator=g, device="cuda")
    _xent_near(q.xent_grad(x, w, t, b, dloss=dloss), x, w, t, b, dloss)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(5, 48, 70), (120, 64, 1000), (600, 40, 30001)])
def test_xent_masked_classes(shape, dtype):
    """Classes taken out by a bias of -inf, or of the lowest value, whole tiles of them
    among them."""
    N, Cs, Ct = shape
    _, x, w, b, t = _xent_case(N, Cs, Ct, dtype)
    cut = Ct // 2
    b[cut:] = -math.inf
    b[0] = torch.finfo(F32).min
    t = t % (cut - 1) + 1
    got = q.xent_grad(x, w, t, b)
    _xent_near(got, x, w, t, b)
    assert not got[3][cut:].any() and not got[4][cut:].any()  # no gradient to what is out
    # a target that is out: an infinite loss, a finite gradient
    t[0] = cut
    loss, lse, dx, dw, db = q.xent_grad(x, w, t, b)
    assert math.isinf(loss[0]) and loss[0] > 0 and bool(torch.isfinite(lse).all())
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
    # no class left: the formula's -inf minus -inf
    loss, lse = q.xent_forward(x, w, t, torch.full((Ct,), -math.inf, device="cuda"))
    assert bool(torch.isnan(loss).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 48, 70), (120, 64, 1000), (600, 40, 30001)])
def test_xent_ignored_rows(shape, dtype):
    """Rows without a class: no loss, no gradient, whatever their x holds, and none of it
    in others'."""
    N, Cs, Ct = shape
    _, x, w, b, t = _xent_case(N, Cs, Ct, dtype)
    clean = q.xent_grad(x[2:].contiguous(), w, t[2:].contiguous(), b)
    t[0], t[1] = -100, -1
    x[0], x[1, 3] = math.nan, math.inf
    loss, lse, dx, dw, db = q.xent_grad(x, w, t, b)
    assert not loss[:2].any() and not dx[:2].any()
    ref, bound = plain.xent(x[2:], w, t[2:], b)
    for a, c, e in zip((loss[2:], lse[2:], dx[2:], dw, db), ref, bound):
        _near(a, c, e)
    for a, c, e in zip(clean, ref, bound):
        _near(a, c, e)
    # all of them, and a class that there is not (taken as none)
    t[:] = -5
    t[N - 1] = Ct
    loss, _, dx, dw, db = q.xent_grad(x, w, t, b)
    assert not loss.any() and not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_xent_strides_alignment_and_order(dtype):
    g = _gen(9)
    for N in (5, 90):
        x, w = _normal(g, N, 67, dtype=dtype, pad=3, off=1), _normal(g, 75, 67, dtype=dtype, pad=1, off=3)
        t = torch.randint(0, 75, (N,), generator=g, device="cuda")
        _xent_near(q.xent_grad(x, w, t), x, w, t, None)


def test_xent_large_logits():
    """Logits of hundreds: no overflow, and the largest class's probability is 1."""
    x = torch.zeros(20, 8, device="cuda")
    x[:, 0] = torch.arange(20, device="cuda") * 50.0
    w = torch.zeros(12, 8, device="cuda")
    w[3, 0], w[4, 0] = 1.0, -1.0
    t = torch.full((20,), 3, device="cuda")
    t[5:] = 4
    _xent_near(q.xent_grad(x, w, t), x, w, t, None)


ORTHO = [(1, 1), (1, 7), (9, 1), (16, 16), (100, 50), (64, 300), (130, 257), (257, 130), (300, 300), (500, 1100),
         (1100, 500)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ORTHO)
def test_orthogonalize(shape, dtype):
    """Against 64 bits, in the norm: the steps multiply what rounding leaves in the small
    singular directions by up to 3.4445 each, 485 in all, and in the others by about one.  X
    has norm 1 when it is first rounded (2^-24 or 2^-17 per element, and eps_sum of each
    product's terms), and the square root of its rank in the end."""
    m, n = shape
    g = _normal(_gen(10), m, n, dtype=dtype, scale=1e-3)
    want = plain.orthogonalize(g)
    got = q.orthogonalize(g)
    unit = 2.0 ** -24 if dtype == F32 else 2.0 ** -17
    sums = (32 + max(m, n) / 16) * 2.0 ** -23 if dtype == BF16 else (32 + max(m, n) / 64) * 2.0 ** -23
    limit = 485 * (unit + sums) * 3 + plain.eps_out(dtype) * float(want.norm())
    assert float((got.double() - want).norm()) <= limit
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalize_options(dtype):
    g = _normal(_gen(11), 60, 90, dtype=dtype, pad=5, off=1)
    for steps in (0, 1, 2, 7):
        want = plain.orthogonalize(g, steps)
        got = q.orthogonalize(g, steps=steps)
        unit = 2.0 ** -24 if dtype == F32 else 2.0 ** -17
        limit = 3.4445 ** steps * 3 * (unit + 40 * 2.0 ** -23) + plain.eps_out(dtype) * float(want.norm())
        assert float((got.double() - want).norm()) <= limit
    want = plain.orthogonalize(g, 3, (1.5, -0.5, 0.0))
    got = q.orthogonalize(g, 3, (1.5, -0.5, 0.0))
    assert float((got.double() - want).norm()) <= 1e-4 + plain.eps_out(dtype) * float(want.norm())
    # in place, with rows apart
    same = q.orthogonalize(g)
    assert q.orthogonalize(g, out=g) is g and torch.equal(g, same)


def test_orthogonalize_scales():
    """The result does not depend on the scale of G, where its norm outweighs eps: squares
    that overflow or vanish in fp32 do not matter."""
    g = _normal(_gen(12), 40, 64)
    want = plain.orthogonalize(g, eps=0)
    limit = 485 * 3 * (2.0 ** -24 + 33 * 2.0 ** -23)
    for s in (1.0, 2.0 ** 60, 2.0 ** 100, 2.0 ** -20):
        assert float((q.orthogonalize(g * s, eps=0).double() - want).norm()) <= limit
    assert not q.orthogonalize(torch.zeros(30, 20, device="cuda"), eps=0).any()
    assert not q.orthogonalize(torch.zeros(30, 20, device="cuda")).any()
    # eps counts: a matrix of norm 1e-7 is halved before the steps
    h = g / g.norm() * 1e-7
    assert float((q.orthogonalize(h, steps=0).double().norm() - 0.5).abs()) < 1e-5
    g[3, 3] = math.nan
    assert bool(torch.isnan(q.orthogonalize(g)).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_repeats_bit_for_bit(dtype):
    g, x, w, b, t = _xent_case(300, 520, 700, dtype)
    dy = _normal(g, 300, 700, dtype=dtype)
    first = [q.dense_forward(x, w, b), *q.dense_backward(dy, x, w), *q.xent_grad(x, w, t, b), q.orthogonalize(w)]
    for _ in range(3):
        again = [q.dense_forward(x, w, b), *q.dense_backward(dy, x, w), *q.xent_grad(x, w, t, b),
                 q.orthogonalize(w)]
        assert all(torch.equal(a, c) for a, c in zip(first, again))


@pytest.mark.parametrize("dtype", TYPES)
def test_other_streams(dtype):
    """Calls on a stream that is not the current one use that stream's memory."""
    g, x, w, b, t = _xent_case(150, 256, 400, dtype)
    want = [q.dense_forward(x, w, b, act="relu"), *q.xent_grad(x, w, t, b), q.orthogonalize(w)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        got = [q.dense_forward(x, w, b, act="relu", stream=side), *q.xent_grad(x, w, t, b, stream=side),
               q.orthogonalize(w, stream=side)]
        noise = [torch.full((150, 400), 3.0, device="cuda") for _ in range(20)]  # the current stream's
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got))
        del noise


def test_in_a_graph():
    _, x, w, b, t = _xent_case(64, 128, 100, F32)
    want = q.xent_grad(x, w, t, b)
    out = q.orthogonalize(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = q.xent_grad(x, w, t, b)
        upd = q.orthogonalize(w)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got)) and torch.equal(out, upd)


@pytest.mark.parametrize("dtype,N", [(F32, 4), (BF16, 4), (F32, 9), (BF16, 9)])
def test_rows_beyond_32_bits(dtype, N):
    """Rows so far apart that offsets pass 2^31 elements."""
    ld = 2 ** 31 // (N - 1) // 8 * 8 + 64
    buf = torch.empty(ld * (N - 1) + 128, dtype=dtype, device="cuda")
    x = buf.as_strided((N, 100), (ld, 1))
    g = _gen(13)
    x.copy_(torch.randn(N, 100, generator=g, device="cuda"))
    w = _normal(g, 64, 100, dtype=dtype)
    y = buf.as_strided((N, 24), (ld, 1), 104)
    want, _, ey, _ = plain.dense_forward(x, w[:24])
    q.dense_forward(x, w[:24], out=y)
    _near(y, want, ey)
    dy = _normal(g, N, 64, dtype=dtype)
    got = q.dense_backward(dy, x, w)
    want, bound = plain.dense_backward(dy, x, w)
    for a, c, e in zip(got, want, bound):
        _near(a, c, e)
    o = q.orthogonalize(x, out=buf.as_strided((N, 100), (ld, 1)))
    assert bool(torch.isfinite(o).all())


@pytest.mark.parametrize("bad", ["dtype", "shape", "columns", "overlap", "bias", "targets", "act", "pre"])
def test_refusals(bad):
    x, w = torch.zeros(12, 16, device="cuda"), torch.zeros(10, 16, device="cuda")
    t = torch.zeros(12, dtype=torch.int64, device="cuda")
    calls = {
        "dtype": [lambda: q.dense_forward(x, w.bfloat16()), lambda: q.dense_forward(x.half(), w.half()),
                  lambda: q.orthogonalize(x.double())],
        "shape": [lambda: q.dense_forward(x, w[:, :8]), lambda: q.dense_forward(x[0], w),
                  lambda: q.dense_backward(x, x, w), lambda: q.dense_forward(x, w, residual=x)],
        "columns": [lambda: q.dense_forward(x.T, torch.zeros(10, 12, device="cuda")),
                    lambda: q.orthogonalize(x[:, ::2])],
        "overlap": [lambda: q.orthogonalize(x.as_strided((4, 16), (8, 1)))],
        "bias": [lambda: q.dense_forward(x, w, torch.zeros(9, device="cuda")),
                 lambda: q.xent_forward(x, w, t, torch.zeros(10, device="cuda").bfloat16())],
        "targets": [lambda: q.xent_forward(x, w, t.int()), lambda: q.xent_grad(x, w, t[:5]),
                    lambda: q.xent_grad(x, w, t, dloss=t)],
        "act": [lambda: q.dense_forward(x, w, act="tanh")],
        "pre": [lambda: q.dense_backward(torch.zeros(12, 10, device="cuda"), x, w, act="relu")],
    }[bad]
    for call in calls:
        with pytest.raises((TypeError, ValueError)):
            call()


def test_debug_build_records_targets():
    """A target of Ct or above is a caller's error, which the debug build records."""
    x, w = torch.randn(20, 16, device="cuda"), torch.randn(10, 16, device="cuda")
    t = torch.zeros(20, dtype=torch.int64, device="cuda")
    q.set_debug(True)
    try:
        q.xent_grad(x, w, t)
        assert q.device_check() == 0
        t[4] = 10
        q.xent_forward(x, w, t)
        assert q.device_check() == 1  # QCNN_CHECK_CODE
        q.dense_backward(x[:, :10].contiguous(), x, w)
        assert q.device_check() == 0
    finally:
        q.set_debug(False)
