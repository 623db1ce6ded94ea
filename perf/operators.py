"""The operators that fine-tune the dense layers of a network: a dense layer with its epilogue and its
backward pass, softmax cross entropy over the classes of a linear layer with its gradient, and the
orthogonalising of an update by Newton-Schulz products.

listed() names the cases, prepare() makes what a program has in hand, run() is one pass: in elementary
torch operations in 32 bits, or (own) by the package's calls.  exact() is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
NS = (3.4445, -4.7750, 2.0315)  # the quintic of the Newton-Schulz steps
EPS = 1e-7


def _dense(name, N, Cs, Ct, dtype, act, residual=False, pre=False):
    return dict(name=name, op="dense_forward", N=N, Cs=Cs, Ct=Ct, dtype=dtype, act=act,
                residual=residual, pre=pre)


def _dense_bwd(name, N, Cs, Ct, dtype, act):
    return dict(name=name, op="dense_backward", N=N, Cs=Cs, Ct=Ct, dtype=dtype, act=act)


def _xent(name, op, N, Cs, Ct, dtype, ignored=0.0, masked=0.0):
    return dict(name=name, op=op, N=N, Cs=Cs, Ct=Ct, dtype=dtype, ignored=ignored, masked=masked)


def _ortho(name, m, n, dtype, steps=5):
    return dict(name=name, op="orthogonalize", m=m, n=n, dtype=dtype, steps=steps)


def listed():
    return [
        # one image through the classifier: latency
        _dense("dense_fwd_fc8_n1_fp32", 1, 4096, 1000, "fp32", "none"),
        # the first FC layer at the benchmark's batch, kept for its backward pass: the weights' bytes
        _dense("dense_fwd_fc6_n128_fp32", 128, 9216, 4096, "fp32", "relu", pre=True),
        # a wide layer with a residual branch on many rows: tensor-core rate
        _dense("dense_fwd_4096_gelu_res_bf16", 4096, 4096, 8192, "bf16", "gelu", residual=True, pre=True),
        # the backward pass of the second FC layer at the benchmark's batch
        _dense_bwd("dense_bwd_fc7_n128_fp32", 128, 4096, 4096, "fp32", "relu"),
        # a ragged batch and an odd width (rows off the 16-byte alignment)
        _dense_bwd("dense_bwd_ragged_bf16", 3001, 2048, 5003, "bf16", "silu"),
        # the loss of an evaluation batch over the 1000 classes
        _xent("xent_fwd_fc8_n128_fp32", "xent_forward", 128, 4096, 1000, "fp32"),
        # the loss and gradient of a training batch, some images without a label
        _xent("xent_grad_fc8_n128_fp32", "xent_grad", 128, 4096, 1000, "fp32", ignored=0.1),
        # a large label set of an odd size, evaluation
        _xent("xent_fwd_50001_bf16", "xent_forward", 1000, 1000, 50001, "bf16", ignored=0.02),
        # the largest: many rows, many classes (the last ones padding, masked by their bias)
        _xent("xent_grad_32768_bf16", "xent_grad", 4096, 2048, 32768, "bf16", ignored=0.05, masked=0.02),
        # updates of a small layer, of the classifier and of the first FC layer
        _ortho("ortho_256x500_fp32", 256, 500, "fp32"),
        _ortho("ortho_fc8_1000x4096_fp32", 1000, 4096, "fp32"),
        _ortho("ortho_fc6_4096x9216_bf16", 4096, 9216, "bf16"),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _most():
    return max(work(c)["flops"] for c in listed())


def draw(rng):
    most = _most()
    while True:
        op = rng.choice(["dense_forward", "dense_backward", "xent_forward", "xent_grad", "orthogonalize"])
        dtype = rng.choice(["fp32", "bf16"])
        if op == "orthogonalize":
            c = _ortho("", _log(rng, 16, 4096), _log(rng, 16, 9216), dtype)
        else:
            N = _log(rng, 1, 4096)
            Cs = _log(rng, 64, 9216)
            if rng.random() < 0.5:  # (widths of layers are mostly round)
                Cs = max(64, Cs // 64 * 64)
            if op.startswith("dense"):
                Ct = _log(rng, 64, 9216)
                act = rng.choice(["none", "relu", "gelu", "silu"])
                if op == "dense_forward":
                    c = _dense("", N, Cs, Ct, dtype, act, rng.random() < 0.5, rng.random() < 0.5)
                else:
                    c = _dense_bwd("", N, Cs, Ct, dtype, act)
            else:
                c = _xent("", op, N, min(Cs, 4096), _log(rng, 64, 50001), dtype,
                          rng.choice([0.0, 0.1]), rng.choice([0.0, 0.02]))
        # fp32 does its operations at a fraction of the rate that the largest case, in bf16, does
        if work(c)["flops"] * (4 if dtype == "fp32" else 1) <= most:
            del c["name"]
            return c


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    dt = TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "orthogonalize":
        # a gradient: a few strong directions above noise
        m, n = case["m"], case["n"]
        r = max(1, min(m, n) // 16)
        s["g"] = (_normal(g, (m, r), 1e-3) @ _normal(g, (r, n), 1 / math.sqrt(r)) +
                  _normal(g, (m, n), 1e-4)).to(dt)
        return s
    N, Cs, Ct = case["N"], case["Cs"], case["Ct"]
    s["x"] = torch.relu(_normal(g, (N, Cs), 1.0)).to(dt)  # activations behind a ReLU
    s["w"] = _normal(g, (Ct, Cs), math.sqrt(2.0 / Cs), dt)
    s["b"] = _normal(g, (Ct,), 0.1)
    if case["op"] == "dense_forward":
        s["r"] = _normal(g, (N, Ct), 1.0, dt) if case["residual"] else None
    elif case["op"] == "dense_backward":
        s["z"] = None if case["act"] == "none" else _normal(g, (N, Ct), 1.0, dt)
        s["dy"] = _normal(g, (N, Ct), 1e-3, dt)
    else:
        s["t"] = torch.randint(0, Ct, (N,), generator=g, device="cuda")
        if case["masked"]:
            k = int(Ct * case["masked"])
            if 0 < k < Ct:
                s["b"][Ct - k:] = -math.inf
                s["t"] %= Ct - k
        if case["ignored"]:
            s["t"][torch.rand((N,), generator=g, device="cuda") < case["ignored"]] = -100
    return s


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _dact(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    sg = 1 / (1 + torch.exp(-z))
    return sg * (1 + z * (1 - sg))


def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    op, dt = c["op"], TYPES[c["dtype"]]
    if op == "orthogonalize":
        x = s["g"].float()
        wide = c["m"] <= c["n"]
        x = x if wide else x.T
        x = x / (torch.sqrt((x * x).sum()) + EPS)
        for _ in range(c["steps"]):
            a = x @ x.T
            x = NS[0] * x + (NS[1] * a + NS[2] * (a @ a)) @ x
        return (x if wide else x.T).to(dt)
    x, w, b = s["x"].float(), s["w"].float(), s["b"]
    if op == "dense_forward":
        z = x @ w.T + b
        y = _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return [y.to(dt), z.to(dt)] if c["pre"] else [y.to(dt)]
    if op == "dense_backward":
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _dact(s["z"].float(), c["act"])
        return [(dz @ w).to(dt), (dz.T @ x).to(dt), dz.sum(0)]
    valid = s["t"] >= 0
    t = torch.where(valid, s["t"], torch.zeros_like(s["t"]))[:, None]
    logits = x @ w.T + b
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    loss = torch.where(valid, (lse - logits.gather(1, t))[:, 0], torch.zeros_like(lse[:, 0]))
    if op == "xent_forward":
        return [loss, lse[:, 0]]
    dl = e / total
    dl.scatter_add_(1, t, -torch.ones_like(lse))
    dl = dl * (valid.float() / valid.sum().clamp(min=1))[:, None]
    return [loss, lse[:, 0], (dl @ w).to(dt), (dl.T @ x).to(dt), dl.sum(0)]


def _own(s, c):
    import paper_1512_06473_gb300 as q
    op = c["op"]
    if op == "orthogonalize":
        return q.orthogonalize(s["g"], steps=c["steps"], eps=EPS)
    if op == "dense_forward":
        y = q.dense_forward(s["x"], s["w"], s["b"], act=c["act"], residual=s["r"], pre=c["pre"])
        return list(y) if c["pre"] else [y]
    if op == "dense_backward":
        return list(q.dense_backward(s["dy"], s["x"], s["w"], pre=s["z"], act=c["act"]))
    if op == "xent_forward":
        return list(q.xent_forward(s["x"], s["w"], s["t"], bias=s["b"]))
    return list(q.xent_grad(s["x"], s["w"], s["t"], bias=s["b"]))


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "orthogonalize":
        p, q = sorted((case["m"], case["n"]))
        # X X^T and A^2 are symmetric: half of each
        return {"bytes": 2 * p * q * e,
                "flops": case["steps"] * (p * (p + 1) * q + p * p * (p + 1) + 2 * p * p * q)}
    N, Cs, Ct = case["N"], case["Cs"], case["Ct"]
    xw, product = (N * Cs + Ct * Cs) * e, 2 * N * Cs * Ct
    if case["op"] == "dense_forward":
        return {"bytes": xw + N * Ct * e * (1 + case["residual"] + case["pre"]) + 4 * Ct, "flops": product}
    if case["op"] == "dense_backward":
        return {"bytes": 2 * xw + N * Ct * e * (1 if case["act"] == "none" else 2) + 4 * Ct,
                "flops": 2 * product}
    if case["op"] == "xent_forward":
        return {"bytes": xw + 4 * Ct + 16 * N, "flops": product}
    return {"bytes": 2 * xw + 8 * Ct + 16 * N, "flops": 3 * product}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalize":
        x = s["g"].double()
        x = x / (torch.linalg.vector_norm(x) + EPS)
        a, b, c = NS
        if case["m"] > case["n"]:  # the same polynomial, of X^T X from the right
            eye = torch.eye(case["n"], dtype=torch.float64, device="cuda")
            for _ in range(case["steps"]):
                gram = x.T @ x
                x = x @ (a * eye + gram @ (b * eye + c * gram))
        else:
            eye = torch.eye(case["m"], dtype=torch.float64, device="cuda")
            for _ in range(case["steps"]):
                gram = x @ x.T
                x = (a * eye + gram @ (b * eye + c * gram)) @ x
        return x
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    if case["op"] == "dense_forward":
        z = torch.addmm(b, x, w.T)
        y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0),
             "gelu": lambda v: v * torch.special.ndtr(v), "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](z)
        if s["r"] is not None:
            y = y + s["r"].double()
        return [y, z] if case["pre"] else [y]
    if case["op"] == "dense_backward":
        dz = s["dy"].double()
        if s["z"] is not None:
            z = s["z"].double()
            if case["act"] == "relu":
                dz = torch.where(z > 0, dz, torch.zeros_like(dz))
            elif case["act"] == "gelu":
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
            else:
                sg = torch.sigmoid(z)
                dz = dz * (sg + z * sg * (1 - sg))
        return [dz @ w, dz.T @ x, dz.sum(0)]
    logits = torch.addmm(b, x, w.T)
    lse = torch.logsumexp(logits, 1)
    keep = s["t"] >= 0
    loss = torch.zeros_like(lse)
    loss[keep] = lse[keep] - logits[keep, s["t"][keep]]
    if case["op"] == "xent_forward":
        return [loss, lse]
    dl = torch.softmax(logits, 1)
    del logits
    dl[keep, s["t"][keep]] -= 1
    dl[~keep] = 0
    dl /= max(1, int(keep.sum()))
    return [loss, lse, dl @ w, dl.T @ x, dl.sum(0)]
