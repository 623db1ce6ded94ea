"""The quantizing of rows and the dense layer in 8-bit integers on the GPU against their plain
forms: codes and scales exactly, products within bounds derived in tests/plain_int8.py."""
import math

import pytest
import torch

import paper_1512_06473_gb300 as q
import plain_int8 as plain
from test_gpu_finetune import _gen, _near, _no_timeouts, _normal

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]
I8 = torch.int8


def _codes(g, rows, cols, low=-127, high=127, pitch=None, off=0):
    """Any codes; pitch: bytes between rows (by default the next multiple of 16)."""
    pitch = (cols + 15) // 16 * 16 if pitch is None else pitch
    room = torch.randint(low, high + 1, (rows * pitch + off,), generator=g, device="cuda", dtype=I8)
    return room[off:].view(rows, pitch)[:, :cols]


def _scales(g, n):
    return torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3


# ---------------------------------------------------------------- quantizer
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (3, 5), (1, 4096), (700, 31), (5, 32), (20, 33), (64, 255), (9, 1000),
                                   (2, 2049), (33, 4097), (4, 9216), (3, 16384), (2, 16385), (2, 40000), (2, 40001),
                                   (5000, 64), (1, 200000)])
def test_quantize(shape, dtype):
    g = _gen(1)
    x = _normal(g, *shape, dtype=dtype) * torch.exp(torch.randn(shape[0], 1, generator=g, device="cuda") * 3).to(dtype)
    codes, scale = q.int8_quantize(x)
    want, s = plain.quantize(x)
    assert codes.dtype == I8 and codes.stride(0) % 16 == 0 and codes.data_ptr() % 16 == 0
    assert torch.equal(scale.cpu(), s)
    assert torch.equal(codes.cpu(), want)
    # what it stands for
    off = (codes.double() * scale.double()[:, None] - x.double()).abs()
    assert bool((off <= (0.5 + 2.0 ** -15) * scale.double()[:, None]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off,pitch", [(0, 1, 0), (1, 0, 1), (3, 2, 5), (8, 0, 16), (8, 4, 8), (16, 8, 4)])
@pytest.mark.parametrize("cols", [16, 100, 2051])
def test_quantize_strides_and_alignment(cols, pad, off, pitch, dtype):
    g = _gen(2)
    x = _normal(g, 11, cols, dtype=dtype, pad=pad, off=off)
    want, s = plain.quantize(x)
    for first in (0, 1, 4, 8):
        room = torch.full((11 * (cols + pitch) + first,), 99, device="cuda", dtype=I8)
        out = room[first:].view(11, cols + pitch)[:, :cols]
        codes, scale = q.int8_quantize(x, out=out)
        assert codes is out and torch.equal(codes.cpu(), want) and torch.equal(scale.cpu(), s)
        rest = room[first:].view(11, cols + pitch)[:, cols:]
        assert bool((rest == 99).all()) and bool((room[:first] == 99).all())


@pytest.mark.parametrize("cols", [7, 64, 3000])
def test_quantize_ties_and_extremes(cols):
    x = torch.zeros(10, cols, device="cuda")
    x[0, 0] = 127.0                              # scale 1 (nearly): halves are ties
    x[0, 1:] = (torch.arange(cols - 1, device="cuda") % 254 - 127) + 0.5
    x[1] = 0.0                                   # the smallest scale
    x[2] = -0.0
    x[3] = torch.finfo(F32).max
    x[3, 1::2] *= -1
    x[4] = 2.0 ** -149
    x[5, 1] = 2.0 ** -120
    x[5, 2] = -2.0 ** -126
    x[6, 3] = float("nan")
    x[7, 4] = float("-inf")
    x[8] = 1.0
    x[8, 2] = float("nan")
    x[8, 3] = float("inf")
    x[9] = -3.0
    codes, scale = q.int8_quantize(x)
    want, s = plain.quantize(x)
    assert torch.equal(codes.cpu(), want)
    assert torch.equal(torch.nan_to_num(scale.cpu(), nan=-1.0), torch.nan_to_num(s, nan=-1.0))
    assert bool(torch.isnan(scale[6])) and bool(torch.isinf(scale[7])) and bool(torch.isnan(scale[8]))
    assert float(scale[1]) == 2.0 ** -126 and int(codes[3, 0]) == 127 and int(codes[3, 1]) == -127


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_of_nothing_and_streams(dtype):
    codes, scale = q.int8_quantize(torch.empty(0, 5, device="cuda", dtype=dtype))
    assert codes.shape == (0, 5) and scale.shape == (0,)
    g = _gen(3)
    x = _normal(g, 300, 1001, dtype=dtype)
    want = q.int8_quantize(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = q.int8_quantize(x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_quantize_beyond_32_bits():
    rows, cols = 70001, 65536
    x = torch.ones(rows, cols, device="cuda", dtype=BF16)
    x[-1] = torch.arange(cols, device="cuda").to(BF16)
    x[32768] *= -2
    codes, scale = q.int8_quantize(x)
    for row in (0, 32767, 32768, 65535, 65536, rows - 1):
        want, s = plain.quantize(x[row:row + 1])
        assert torch.equal(codes[row].cpu(), want[0]) and float(scale[row]) == float(s[0])
    del x, codes
    torch.cuda.empty_cache()


# -------------------------------------------------------------- dense layer
DENSE = [  # N, Cs, Ct: few rows, one tile, ragged tiles, blocks of 1024 terms, several tiles, split sums
    (1, 1, 1), (1, 15, 3), (1, 64, 64), (1, 4096, 1000), (1, 9216, 130), (2, 100, 33), (3, 17, 5), (4, 1000, 999),
    (5, 1001, 7), (8, 520, 130), (8, 4096, 513), (9, 64, 16), (9, 4000, 300), (16, 128, 128), (17, 33, 65),
    (31, 2048, 200), (33, 2000, 1), (64, 129, 64), (65, 1024, 129), (100, 72, 200), (128, 4096, 256),
    (129, 300, 127), (130, 1, 140), (200, 9216, 128), (255, 1025, 131), (257, 64, 513), (300, 515, 301),
    (300, 5000, 2000), (700, 1024, 640), (1025, 1100, 700), (2000, 200, 1500), (8, 9000, 5000), (64, 131071, 9),
    (3, 131071, 40)]


def _dense_case(seed, N, Cs, Ct, codes, dtype, **kw):
    g = _gen(seed)
    w, ws = _codes(g, Ct, Cs, **kw), _scales(g, Ct)
    if codes:
        x, xs = _codes(g, N, Cs, **kw), _scales(g, N)
        return g, x, xs, w, ws, (x, xs)
    x = _normal(g, N, Cs, dtype=dtype)
    c, s = plain.quantize(x)
    return g, x, None, w, ws, (c.cuda(), s.cuda())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("shape", DENSE)
def test_dense(shape, codes, dtype):
    N, Cs, Ct = shape
    g, x, xs, w, ws, (c, s) = _dense_case(1, N, Cs, Ct, codes, dtype)
    b = torch.randn(Ct, generator=g, device="cuda")
    y = q.int8_dense_forward(x, w, ws, b, xscale=xs, dtype=dtype)
    assert y.dtype == dtype
    want, bound = plain.dense(c, s, w, ws, b)
    _near(y, want, bound)
    _no_timeouts()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(3, 70, 90), (12, 640, 300), (150, 200, 144), (140, 2000, 301), (600, 1500, 520)])
def test_dense_epilogues(shape, act, dtype):
    N, Cs, Ct = shape
    g, x, _, w, ws, (c, s) = _dense_case(2, N, Cs, Ct, False, dtype)
    b, r = torch.randn(Ct, generator=g, device="cuda"), _normal(g, N, Ct, dtype=dtype)
    y = q.int8_dense_forward(x, w, ws, b, act=act, residual=r)
    _near(y, *plain.dense(c, s, w, ws, b, act, r))
    # the residual's memory may be the output's
    out = r.clone()
    assert torch.equal(q.int8_dense_forward(x, w, ws, b, act=act, residual=out, out=out), y)
    # no bias; codes by hand are the call's own
    plain_y = q.int8_dense_forward(x, w, ws, act=act)
    _near(plain_y, *plain.dense(c, s, w, ws, None, act))
    own = q.int8_quantize(x)
    assert torch.equal(q.int8_dense_forward(own[0], w, ws, act=act, xscale=own[1], dtype=dtype), plain_y)


@pytest.mark.parametrize("N", [1, 4, 8, 40, 300])
@pytest.mark.parametrize("pitch,off", [(0, 0), (0, 1), (1, 0), (16, 0), (16, 8), (7, 3)])
@pytest.mark.parametrize("cols", [48, 131, 1031])
def test_dense_strides_and_alignment(cols, pitch, off, N):
    g = _gen(3)
    w, ws = _codes(g, 77, cols, pitch=cols + pitch, off=off), _scales(g, 77)
    x, xs = _codes(g, N, cols, pitch=cols + pitch, off=off), _scales(g, N)
    room = torch.full((N, 77 + pitch), 7.0, device="cuda")
    r = _normal(g, N, 77, pad=pitch, off=off)
    y = q.int8_dense_forward(x, w, ws, residual=r, xscale=xs, out=room[:, :77])
    _near(y, *plain.dense(x, xs, w, ws, None, "none", r))
    assert bool((room[:, 77:] == 7).all())  # nothing between the rows is written
    f = _normal(g, N, cols, pad=pitch, off=off)
    c, s = plain.quantize(f)
    half = torch.full((N, 77 + pitch), 7.0, device="cuda", dtype=BF16)
    q.int8_dense_forward(f.to(BF16), w, ws, out=half[:, :77])
    c, s = plain.quantize(f.to(BF16))
    _near(half[:, :77], *plain.dense(c.cuda(), s.cuda(), w, ws))
    assert bool((half[:, 77:] == 7).all())
    _no_timeouts()


@pytest.mark.parametrize("N", [1, 8, 9, 40, 200])
@pytest.mark.parametrize("Cs", [1000, 1024, 2048, 9216])
def test_sums_of_codes_are_exact(Cs, N):
    """Sums below 2^24 come out exactly, whatever the codes: of 1024 products of -128, of odd sums near
    the end of what 24 bits hold, of blocks that cancel."""
    g = _gen(4)
    Ct = 140
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    for low, high, keep in ((-128, 127, None), (90, 127, 1023), (-128, -120, 1000)):
        x, w = _codes(g, N, Cs, low, high), _codes(g, Ct, Cs, low, high)
        if keep is not None:  # (1023 terms: below 2^24)
            x[:, keep:] = 0
        y = q.int8_dense_forward(x, w, one(Ct), xscale=one(N))
        want = x.double() @ w.double().T
        assert float(want.abs().max()) < 2 ** 24
        assert torch.equal(y.double(), want)
    # a block of the largest sums, then one that takes it back but for an odd rest
    x, w = torch.full((N, Cs), -128, device="cuda", dtype=I8), torch.full((Ct, Cs), -128, device="cuda", dtype=I8)
    if Cs >= 2048:
        w[:, 1024:2048] = 127
        x[:, 2048:] = 0
    elif Cs == 1024:
        x[:, 1000:] = 1
    y = q.int8_dense_forward(x, w, one(Ct), xscale=one(N))
    assert torch.equal(y.double(), x.double() @ w.double().T)


@pytest.mark.parametrize("N", [2, 100])
def test_largest_sums(N):
    x = torch.full((N, 131071), -128, device="cuda", dtype=I8)
    w = torch.full((130, 131071), -128, device="cuda", dtype=I8)
    w[1::2] = 127
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    y = q.int8_dense_forward(x, w, one(130), xscale=one(N))
    _near(y, *plain.dense(x, one(N), w, one(130)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [3, 60])
def test_non_finite_rows(N, dtype):
    g = _gen(5)
    x = _normal(g, N, 200, dtype=dtype)
    x[0, 3] = float("nan")
    x[1, 199] = float("inf")
    wd = _normal(g, 70, 200)
    wd[5, 5] = float("inf")
    w, ws = q.int8_quantize(wd)
    y = q.int8_dense_forward(x, w, ws)
    assert not bool(torch.isfinite(y[:2]).any()) and not bool(torch.isfinite(y[:, 5]).any())
    fine = torch.ones(70, dtype=torch.bool, device="cuda")
    fine[5] = False
    assert bool(torch.isfinite(y[2:, fine]).all())
    # of an empty row (all zero) the bias is left
    x = torch.zeros(N, 200, device="cuda", dtype=dtype)
    b = _normal(g, 1, 70)[0].contiguous()
    w, ws = q.int8_quantize(_normal(g, 70, 200))
    assert torch.equal(q.int8_dense_forward(x, w, ws, b), b.to(dtype).expand(N, 70))


@pytest.mark.parametrize("N", [2, 50])
def test_scales_at_the_ends_of_the_range(N):
    # a product of two scales may leave fp32's range where the result does not
    g = _gen(6)
    w, x = _codes(g, 40, 300), _codes(g, N, 300)
    for a, b in ((1e-30, 1e30), (1e30, 1e-30), (2.0 ** -126, 1.0), (1e-20, 1e-18)):
        ws, xs = torch.full((40,), b, device="cuda"), torch.full((N,), a, device="cuda")
        _near(q.int8_dense_forward(x, w, ws, xscale=xs), *plain.dense(x, xs, w, ws))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1, 8, 30, 500])
def test_streams_graphs_and_repeats(N, dtype):
    g = _gen(7)
    x = _normal(g, N, 1500, dtype=dtype)
    w, ws = q.int8_quantize(_normal(g, 700, 1500))
    want = q.int8_dense_forward(x, w, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [q.int8_dense_forward(x, w, ws, stream=s) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(v, want) for v in got)
    # two graphs that share a workspace and run one after another
    from paper_1512_06473_gb300 import _lib, _scratch
    nb = _scratch(_lib.load(), "qcnn_int8_dense_workspace_size", N, 1500, 700, 0, 1)
    room = torch.empty(nb + 256, device="cuda", dtype=torch.uint8)
    room = room[-room.data_ptr() % 256:][:max(nb, 1)]
    x2 = x.clone()
    outs, graphs = [torch.empty_like(want) for _ in range(2)], []
    for v, out in zip((x, x2), outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            q.int8_dense_forward(v, w, ws, out=out, workspace=room)
        graphs.append(graph)
    x2.neg_()
    for graph in graphs + graphs[::-1]:
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)
    assert torch.equal(outs[1], q.int8_dense_forward(x2, w, ws))


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    w, ws = torch.zeros(3, 16, device="cuda", dtype=I8), torch.ones(3, device="cuda")
    assert q.int8_dense_forward(torch.empty(0, 16, device="cuda", dtype=dtype), w, ws).shape == (0, 3)


def test_many_outputs_and_rows():
    # more than 2^31 outputs' elements; rows that are checked lie at both ends
    g = _gen(8)
    N, Cs, Ct = 40000, 32, 60000
    x, xs, w, ws = _codes(g, N, Cs), _scales(g, N), _codes(g, Ct, Cs), _scales(g, Ct)
    y = q.int8_dense_forward(x, w, ws, xscale=xs, dtype=BF16)
    for rows in (slice(0, 3), slice(35790, 35800), slice(N - 3, N)):
        _near(y[rows], *plain.dense(x[rows], xs[rows], w, ws))
    del y
    torch.cuda.empty_cache()
    _no_timeouts()


def test_close_to_the_dense_layer():
    """The layer that the codes stand for, within what quantizing loses: half a step of each operand."""
    g = _gen(9)
    x, wd = torch.relu(_normal(g, 100, 1000)), _normal(g, 300, 1000, scale=1 / math.sqrt(1000))
    w, ws = q.int8_quantize(wd)
    y, dense = q.int8_dense_forward(x, w, ws).double(), q.dense_forward(x, wd).double()
    _, xs = q.int8_quantize(x)
    half = 0.5 + 2.0 ** -15
    bound = half * (x.double().abs().sum(1)[:, None] * ws.double() + xs.double()[:, None] * wd.double().abs().sum(1)) \
        + half ** 2 * 1000 * xs.double()[:, None] * ws.double() + 1e-4
    assert bool(((y - dense).abs() <= bound).all())
