"""Dropout while the dense layers of a network are trained, and the same layers in 8-bit integers
once they are: dropout from a counter-based generator whose mask is never stored, with its gradient;
the quantising of a matrix row by row; and a dense layer on 8-bit weights with a scale per output and
inputs with a scale per row.

listed() names the cases, prepare() makes what a program has in hand, run() is one pass: in elementary
torch operations in 32 bits, or (own) by the package's calls.  exact() is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
LEAST = 2.0 ** -126        # the smallest scale of a row
STEP = 0x810204 * 2.0 ** -30  # 1 / 127 in 32 bits


def _dropout(name, op, rows, cols, dtype, p, residual=False, counter=False):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, counter=counter)


def _quantize(name, rows, cols, dtype):
    return dict(name=name, op="int8_quantize", rows=rows, cols=cols, dtype=dtype)


def _dense(name, N, Cs, Ct, dtype, act="none", residual=False, codes=False):
    return dict(name=name, op="int8_dense", N=N, Cs=Cs, Ct=Ct, dtype=dtype, act=act, residual=residual, codes=codes)


def listed():
    return [
        # behind the second FC layer's ReLU in a training step at the benchmark's batch: latency
        _dropout("dropout_fwd_128x4096_fp32", "dropout_forward", 128, 4096, "fp32", 0.5),
        # many rows of a wide layer on a residual branch, as a captured training step runs it (the
        # generator's offset in device memory): the bytes
        _dropout("dropout_fwd_16384x9216_res_bf16", "dropout_forward", 16384, 9216, "bf16", 0.1, True, True),
        # the gradient on the way to the second FC layer
        _dropout("dropout_bwd_128x4096_fp32", "dropout_backward", 128, 4096, "fp32", 0.5),
        # a ragged batch and an odd width
        _dropout("dropout_bwd_3001x5003_bf16", "dropout_backward", 3001, 5003, "bf16", 0.2, counter=True),
        # the first FC layer's weights, once they are trained
        _quantize("quantize_fc6_4096x9216_fp32", 4096, 9216, "fp32"),
        # a ragged batch's activations of an odd width, quantized once for several layers
        _quantize("quantize_rows_1000x4097_bf16", 1000, 4097, "bf16"),
        # one image through the classifier: latency
        _dense("int8_fc8_n1_fp32", 1, 4096, 1000, "fp32"),
        # one image through the first FC layer: the weights' bytes
        _dense("int8_fc6_n1_bf16", 1, 9216, 4096, "bf16", "relu"),
        # a few images at once
        _dense("int8_fc7_n8_bf16", 8, 4096, 4096, "bf16", "relu"),
        # the first FC layer at the benchmark's batch
        _dense("int8_fc6_n128_fp32", 128, 9216, 4096, "fp32", "relu"),
        # a ragged batch that comes quantized, odd widths
        _dense("int8_ragged_codes_fp32", 3001, 2047, 5003, "fp32", codes=True),
        # many rows of a wide layer with a residual branch: tensor-core rate
        _dense("int8_4096_gelu_res_bf16", 4096, 4096, 8192, "bf16", "gelu", residual=True),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["dropout_forward", "dropout_backward", "int8_quantize", "int8_dense", "int8_dense"])
        dtype = rng.choice(["fp32", "bf16"])
        if op.startswith("dropout"):
            c = _dropout("", op, _log(rng, 1, 16384), _log(rng, 16, 9216), dtype, rng.choice([0.1, 0.2, 0.5]),
                         op == "dropout_forward" and rng.random() < 0.5, rng.random() < 0.5)
        elif op == "int8_quantize":
            c = _quantize("", _log(rng, 1, 8192), _log(rng, 16, 9216), dtype)
        else:
            Cs = _log(rng, 64, 9216)
            if rng.random() < 0.5:  # (widths of layers are mostly round)
                Cs = max(64, Cs // 64 * 64)
            c = _dense("", _log(rng, 1, 4096), Cs, _log(rng, 64, 9216), dtype,
                       rng.choice(["none", "relu", "gelu", "silu"]), rng.random() < 0.5, rng.random() < 0.25)
        if all(work(c)[k] <= most[k] for k in most):
            del c["name"]
            return c


def _normal(g, shape, std, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _codes_of(x):
    """(codes, scales) of the rows of x, each step in 32 bits: s = max |x| (1 / 127), and the whole
    number nearest to x (1 / s), ties to even."""
    x = x.float()
    s = (x.abs().amax(1) * STEP).clamp(min=LEAST)
    q = torch.round(x * torch.reciprocal(s)[:, None]).clamp(-127, 127)
    return q.to(torch.int8), s


def _held(codes):
    """Codes as a program keeps them: rows 16-byte multiples apart."""
    rows, cols = codes.shape
    room = torch.zeros((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=codes.device)
    room[:, :cols] = codes
    return room[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"].startswith("dropout"):
        rows, cols = case["rows"], case["cols"]
        if case["op"] == "dropout_forward":
            s["x"] = torch.relu(_normal(g, (rows, cols), 1.0)).to(dt)  # behind a ReLU
            s["r"] = _normal(g, (rows, cols), 1.0, dt) if case["residual"] else None
        else:
            s["x"] = _normal(g, (rows, cols), 1e-3, dt)
        s["seed"] = 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 62)
        s["offset"] = 5 + seed % 1000
        if case["counter"]:
            s["offset"] = torch.tensor([s["offset"] + (1 << 33)], device="cuda")
        return s
    if case["op"] == "int8_quantize":
        # rows of different sizes, as the outputs of a trained layer have them
        s["x"] = (_normal(g, (case["rows"], case["cols"]), 0.02) *
                  torch.exp(_normal(g, (case["rows"], 1), 0.5))).to(dt)
        return s
    N, Cs, Ct = case["N"], case["Cs"], case["Ct"]
    w, s["ws"] = _codes_of(_normal(g, (Ct, Cs), math.sqrt(2.0 / Cs)))
    s["w"] = _held(w)
    s["b"] = _normal(g, (Ct,), 0.1)
    x = torch.relu(_normal(g, (N, Cs), 1.0))
    if case["codes"]:
        x, s["xs"] = _codes_of(x)
        s["x"] = _held(x)
    else:
        s["x"], s["xs"] = x.to(dt), None
    s["r"] = _normal(g, (N, Ct), 1.0, dt) if case["residual"] else None
    return s


def _philox(seed, offset, n, device):
    """The n 32-bit words of the generator of counters (i, 0, offset) and the key `seed`, four to a
    counter: Philox-4x32 with ten rounds (Salmon et al. 2011), in 64-bit integers."""
    low = 0xFFFFFFFF
    i = torch.arange((n + 3) // 4, device=device)
    c0, c1 = i & low, i >> 32
    if torch.is_tensor(offset):
        c2, c3 = (offset & low).expand_as(i), (offset >> 32 & low).expand_as(i)
    else:
        c2, c3 = torch.full_like(i, offset & low), torch.full_like(i, offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # (the low 64 bits, in a signed integer)
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], 1).view(-1)[:n]


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    op, dt, x = c["op"], TYPES[c["dtype"]], s["x"]
    if op.startswith("dropout"):
        keep = (_philox(s["seed"], s["offset"], x.numel(), x.device) >= round(c["p"] * 2.0 ** 32)).view(x.shape)
        y = torch.where(keep, x.float() * (1 / (1 - c["p"])), torch.zeros((), device=x.device))
        if op == "dropout_forward" and s["r"] is not None:
            y = y + s["r"].float()
        return [y.to(dt)]
    if op == "int8_quantize":
        return list(_codes_of(x))
    q, xs = (x, s["xs"]) if c["codes"] else _codes_of(x)
    z = (q.float() @ s["w"].float().T) * s["ws"] * xs[:, None] + s["b"]
    y = _act(z, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return [y.to(dt)]


def _own(s, c):
    import paper_1512_06473_gb300 as q
    op = c["op"]
    if op == "dropout_forward":
        return [q.dropout_forward(s["x"], c["p"], s["seed"], s["offset"], residual=s["r"])]
    if op == "dropout_backward":
        return [q.dropout_backward(s["x"], c["p"], s["seed"], s["offset"])]
    if op == "int8_quantize":
        return list(q.int8_quantize(s["x"]))
    return [q.int8_dense_forward(s["x"], s["w"], s["ws"], s["b"], act=c["act"], residual=s["r"], xscale=s["xs"],
                                 dtype=TYPES[c["dtype"]])]


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["op"].startswith("dropout"):
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (2 + case["residual"]), "flops": 2 * n}
    if case["op"] == "int8_quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (e + 1) + 4 * case["rows"], "flops": 2 * n}
    N, Cs, Ct = case["N"], case["Cs"], case["Ct"]
    return {"bytes": N * Cs * (1 if case["codes"] else e) + Ct * Cs + N * Ct * e * (1 + case["residual"]) + 8 * Ct +
            (4 * N if case["codes"] else 0), "flops": 2 * N * Cs * Ct}


def _words(seed, offset, n, device):
    """The generator once more, as numbers of 16 bits whose products a double holds."""
    i = torch.arange((n + 3) // 4, device=device)
    v = [i % 2 ** 32, i // 2 ** 32, torch.full_like(i, offset % 2 ** 32), torch.full_like(i, offset // 2 ** 32)]
    k = [seed % 2 ** 32, seed // 2 ** 32]

    def times(m, x):  # (high, low) halves of m x
        lo = x % 65536 * m            # below 2^48
        hi = x // 65536 * m + lo // 65536
        return hi // 65536, hi % 65536 * 65536 + lo % 65536
    for r in range(10):
        h0, l0 = times(3528531795, v[0])
        h1, l1 = times(3449720151, v[2])
        v = [h1 ^ v[1] ^ ((k[0] + r * 2654435769) % 2 ** 32), l1, h0 ^ v[3] ^ ((k[1] + r * 3144134277) % 2 ** 32), l0]
    out = torch.empty((i.numel(), 4), dtype=torch.int64, device=device)
    for j in range(4):
        out[:, j] = v[j]
    return out.flatten()[:n]


def _rounded_codes(x):
    """Codes as defined (each step rounded to 32 bits, here from 64), and scales in 64 bits."""
    x = x.double()
    top = x.abs().max(1).values
    s = torch.maximum(top * STEP, torch.full_like(top, LEAST)).float().double()
    codes = torch.round((x * torch.reciprocal(s).float().double()[:, None]).float().double()).clamp(-127, 127)
    return codes, torch.maximum(top / 127, torch.full_like(top, LEAST))


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"]
    if case["op"].startswith("dropout"):
        words = _words(s["seed"], int(s["offset"]), x.numel(), x.device).view(x.shape)
        y = x.double() / (1 - case["p"])
        y[words < round(case["p"] * 2 ** 32)] = 0
        if case["op"] == "dropout_forward" and s["r"] is not None:
            y += s["r"].double()
        return [y]
    if case["op"] == "int8_quantize":
        q, scales = _rounded_codes(x)
        return [q.to(torch.int8), scales]
    q, scales = (x.double(), s["xs"].double()) if case["codes"] else _rounded_codes(x)
    z = torch.addmm(s["b"].double(), q * scales[:, None], (s["w"].double() * s["ws"].double()[:, None]).T)
    y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * torch.special.ndtr(v),
         "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](z)
    return [y if s["r"] is None else y + s["r"].double()]
