"""The 8-bit dense layer's tiles on the tensor cores, and where its routes change: every tile width,
shares of a tile's terms, pairs of CTAs, ragged edges, results that pass through shared memory and those
that cannot, sums that have to be drained on the way."""
import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _no_timeouts, _normal
from test_gpu_int8 import _codes, _scales

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]
I8 = torch.int8

TILES = [  # N, Cs, Ct
    (16, 9216, 4096), (8, 5121, 100), (257, 64, 513), (33, 9216, 130), (128, 1024, 1029), (700, 1024, 640),
    (129, 1000, 1024), (1025, 1100, 700), (200, 9216, 1000), (300, 2048, 1000), (300, 5000, 2001), (601, 4097, 3001),
    (2000, 200, 1500), (2049, 1025, 1537), (1999, 3000, 1535), (3001, 2047, 5003), (1000, 1000, 4000), (1999, 9216, 2001),
    (3000, 12000, 1000)]


def _case(seed, N, Cs, Ct, codes, dtype, low=-127, high=127):
    g = _gen(seed)
    w, ws = _codes(g, Ct, Cs, low, high), _scales(g, Ct)
    if codes:
        x, xs = _codes(g, N, Cs, low, high), _scales(g, N)
        return g, x, xs, w, ws, (x, xs)
    x = _normal(g, N, Cs, dtype=dtype)
    c, s = plain.quantize(x)
    return g, x, None, w, ws, (c.cuda(), s.cuda())


def test_every_route_is_among_them():
    routes = [q.int8_route(*t) for t in TILES]
    assert not any(r["few"] for r in routes)
    assert {r["rows"] for r in routes} == {16, 32, 64, 128, 160, 192, 224, 256}
    assert {r["shares"] for r in routes} == {1, 2, 4, 8}
    assert all((r["ctas"] == 2) == (r["rows"] > 128) for r in routes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("shape", TILES)
def test_tiles(shape, codes, dtype):
    N, Cs, Ct = shape
    g, x, xs, w, ws, (c, s) = _case(1, N, Cs, Ct, codes, dtype)
    b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    _near(q.int8_dense_forward(x, w, ws, b, xscale=xs, dtype=dtype), *plain.dense(c, s, w, ws, b))
    y = q.int8_dense_forward(x, w, ws, b, act="relu", residual=r, xscale=xs, dtype=dtype)
    _near(y, *plain.dense(c, s, w, ws, b, "relu", r))
    out = r.clone()
    assert torch.equal(q.int8_dense_forward(x, w, ws, b, act="relu", residual=out, out=out, xscale=xs, dtype=dtype), y)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("shape", [(40, 300, 4000), (300, 2048, 1000), (2000, 1500, 1500)])
def test_activations(shape, act, dtype):
    N, Cs, Ct = shape
    g, x, xs, w, ws, (c, s) = _case(2, N, Cs, Ct, False, dtype)
    ws = ws * 0.01
    b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    b[:8] = torch.tensor([30.0, -30.0, 1e4, -1e4, 5.5, -5.5, 0.0, -0.0], device="cuda")
    _near(q.int8_dense_forward(x, w, ws, b, act=act), *plain.dense(c, s, w, ws, b, act))
    _near(q.int8_dense_forward(x, w, ws, b, act=act, residual=r), *plain.dense(c, s, w, ws, b, act, r))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off", [(0, 1), (1, 0), (4, 0), (8, 8), (2, 4)])
@pytest.mark.parametrize("shape", [(40, 300, 4000), (300, 2048, 1000), (2000, 300, 1500), (2000, 300, 1504),
                                   (1000, 1200, 3002)])
def test_results_and_residuals_of_any_alignment(shape, pad, off, dtype):
    N, Cs, Ct = shape
    g, x, xs, w, ws, (c, s) = _case(3, N, Cs, Ct, False, dtype)
    r = _normal(g, N, Ct, dtype=dtype, pad=pad, off=off)
    want = plain.dense(c, s, w, ws, None, "none", r)
    flat = torch.full((N * (Ct + pad) + off,), 7.0, device="cuda", dtype=dtype)
    room = flat[off:].view(N, Ct + pad)
    q.int8_dense_forward(x, w, ws, residual=r, out=room[:, :Ct])
    _near(room[:, :Ct], *want)
    assert bool((room[:, Ct:] == 7).all()) and bool((flat[:off] == 7).all())
    # one of the two alone
    _near(q.int8_dense_forward(x, w, ws, residual=r), *want)
    room.fill_(7.0)
    q.int8_dense_forward(x, w, ws, residual=r.contiguous(), out=room[:, :Ct])
    _near(room[:, :Ct], *want)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("pitch,off", [(0, 3), (1, 0), (16, 8), (16, 16)])
@pytest.mark.parametrize("shape", [(300, 2047, 1000), (2000, 1131, 1500)])
def test_weights_and_codes_of_any_alignment(shape, pitch, off, codes):
    N, Cs, Ct = shape
    g = _gen(4)
    w, ws = _codes(g, Ct, Cs, pitch=Cs + pitch, off=off), _scales(g, Ct)
    if codes:
        x, xs = _codes(g, N, Cs, pitch=Cs + pitch, off=off), _scales(g, N)
        _near(q.int8_dense_forward(x, w, ws, xscale=xs), *plain.dense(x, xs, w, ws))
    else:
        x = _normal(g, N, Cs, pad=pitch, off=off)
        c, s = plain.quantize(x)
        _near(q.int8_dense_forward(x, w, ws), *plain.dense(c.cuda(), s.cuda(), w, ws))


@pytest.mark.parametrize("shape", [(300, 1024, 1000), (300, 5000, 2001), (601, 9216, 3001), (1999, 3000, 1535),
                                   (1500, 9216, 1301), (2300, 9216, 2100), (600, 131071, 2001), (2304, 131071, 2048)])
def test_sums_are_exact(shape):
    """Sums below 2^24 in magnitude come out exactly, whatever is summed on the way."""
    N, Cs, Ct = shape
    g = _gen(5)
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    for low, high in ((-128, 127), (100, 127)):
        x, w = _codes(g, N, Cs, low, high), _codes(g, Ct, Cs, low, high)
        if low > 0:  # large sums that cancel, term for term but the last ones
            half = (Cs - 11) // 2
            x[:, half:2 * half] = -x[:, :half]
            w[:, half:2 * half] = w[:, :half]
        want = x.double() @ w.double().T
        assert float(want.abs().max()) < 2 ** 24
        y = q.int8_dense_forward(x, w, one(Ct), xscale=one(N))
        assert torch.equal(y.double(), want)
    # every product the largest there is, of both signs by blocks of 1024
    x = torch.full((N, Cs), -128, device="cuda", dtype=I8)
    w = torch.full((Ct, Cs), -128, device="cuda", dtype=I8)
    for block in (1, 3):
        w[:, 1024 * block:1024 * block + 1024] = 127
    w[:, 4096:] = 1
    y = q.int8_dense_forward(x, w, one(Ct), xscale=one(N))
    assert torch.equal(y.double(), x.double() @ w.double().T)


def test_rows_that_fill_a_sum_share_a_tile_with_rows_that_do_not():
    N, Cs, Ct = 1999, 5000, 1535
    g = _gen(6)
    x, w = _codes(g, N, Cs, -3, 3), _codes(g, Ct, Cs)
    x[[0, 255, 256, 700, N - 1]] = 127
    x[701, 1024:2048] = -128
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    y = q.int8_dense_forward(x, w, one(Ct), xscale=one(N))
    assert torch.equal(y.double(), x.double() @ w.double().T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(300, 2048, 1000), (2000, 1500, 1500)])
def test_non_finite_rows(shape, dtype):
    N, Cs, Ct = shape
    g, x, _, w, ws, (c, s) = _case(7, N, Cs, Ct, False, dtype)
    x[1, 3] = float("nan")
    x[257, Cs - 1] = float("-inf")
    ws[5] = float("inf")
    for act in ("none", "relu", "gelu", "silu"):
        y = q.int8_dense_forward(x, w, ws, act=act)
        finite = torch.isfinite(y)
        assert not bool(finite[1].any()) and not bool(finite[257].any())
        rest = torch.ones(N, dtype=torch.bool, device="cuda")
        rest[[1, 257]] = False
        keep = torch.arange(Ct, device="cuda") != 5
        assert bool(finite[rest][:, keep].all())
        if act == "none":
            assert not bool(finite[:, 5].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(3, 70, 90), (300, 2048, 1000), (2000, 1500, 1500), (2000, 300, 1501)])
def test_infinite_sums_keep_what_the_activations_make_of_them(shape, dtype):
    """Biases of infinities, and sums at fp32's end: z Phi(z) and z / (1 + exp(-z)) on every route."""
    N, Cs, Ct = shape
    g, x, _, w, ws, (c, s) = _case(10, N, Cs, Ct, False, dtype)
    b = torch.zeros(Ct, device="cuda")
    b[:4] = torch.tensor([float("inf"), float("-inf"), 3.3e38, -3.3e38], device="cuda")
    for act in ("none", "relu", "gelu", "silu"):
        y = q.int8_dense_forward(x, w, ws, b, act=act)
        assert bool((y[:, 0] == float("inf")).all())
        if act == "relu":
            assert bool((y[:, 1] == 0).all())
        elif act != "none":
            assert bool(torch.isnan(y[:, 1]).all())  # (-inf times 0, as in the formulas)
        top = 3.3e38 if dtype == F32 else float(torch.tensor(3.3e38).to(BF16))
        assert bool(((y[:, 2].double() / top - 1).abs() <= 2.0 ** -7).all())
        if act != "none":
            assert bool((y[:, 3] == 0).all())
        assert bool(torch.isfinite(y[:, 4:]).all())


@pytest.mark.parametrize("N,Cs,Ct", [(8, 5120, 500), (9, 5120, 400), (64, 1024, 1831), (128, 900, 1024), (1000, 100, 131),
                                     (4096, 16, 32), (65535, 3, 2), (131072, 1, 1)])
def test_few_terms_and_outputs_of_many_rows(N, Cs, Ct):
    assert q.int8_route(N, Cs, Ct)["few"]
    for dtype in TYPES:
        g, x, xs, w, ws, (c, s) = _case(8, N, Cs, Ct, N % 2 == 0, dtype)
        b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype, pad=3)
        y = q.int8_dense_forward(x, w, ws, b, act="gelu", residual=r, xscale=xs, dtype=dtype)
        _near(y, *plain.dense(c, s, w, ws, b, "gelu", r))


@pytest.mark.parametrize("N", [300, 1999])
def test_two_streams_at_once(N):
    g = _gen(9)
    x = [_normal(g, N, 3000, dtype=BF16) for _ in range(2)]
    w, ws = q.int8_quantize(_normal(g, 1535, 3000))
    want = [q.int8_dense_forward(v, w, ws) for v in x]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(q.int8_dense_forward(x[i], w, ws))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(v, want[i]) for v in got[i])
    _no_timeouts()
