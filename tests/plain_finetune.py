"""Plain 64-bit forms of the fine-tuning operators (torch, any device), and bounds on what
fp32 sums and roundings to fp32 or bf16 may differ from them by.

Bounds, per element.  A sum of K products p_k that is kept in fp32 differs from the exact
one by at most eps_sum(K) * sum |p_k|:
  bf16 operands: products exact, added 16 at a time to an fp32 sum that may be cut off
    instead of rounded (2^-23 of the sum each time), or one by one with rounding (2^-24):
    (K / 16 + 8) 2^-23, or K 2^-24 / (lanes that share it) which is less;
  fp32 operands: three bf16 pieces leave out products below 3 * 2^-24 of each term; six
    products of 16 terms each are added to a sum of 64 terms (24 cut-offs at most), whose
    sums are added with rounding (K / 64), and those of up to 64 splits;
    (32 + K / 64) 2^-23 covers both.
A result is then rounded once: 2^-p of it, p = 24 (fp32) or 8 (bf16) significant bits.
"""
import math

import torch

NS = (3.4445, -4.7750, 2.0315)


def eps_sum(K, dtype):
    return (K / 16 + 8) * 2.0 ** -23 if dtype == torch.bfloat16 else (32 + K / 64) * 2.0 ** -23


def eps_out(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def dense_forward(x, w, b=None, name="none", r=None):
    """(y, z) in 64 bits, and the bounds of their fp32 forms before the last rounding."""
    dt = x.dtype
    x, w = x.double(), w.double()
    z = x @ w.T
    mag = x.abs() @ w.abs().T
    if b is not None:
        z = z + b.double()
        mag = mag + b.double().abs()
    ez = eps_sum(x.shape[1], dt) * mag + 2.0 ** -24 * z.abs()
    y = act(z, name)
    # |act'| <= 1.13; erf and exp in fp32 are good to a few units of 2^-23
    ey = 1.13 * ez + 8 * 2.0 ** -23 * (z.abs() if name in ("gelu", "silu") else 0 * z)
    if r is not None:
        y = y + r.double()
        ey = ey + 2.0 ** -24 * y.abs()
    return y, z, ey, ez


def dense_backward(dy, x, w, z=None, name="none"):
    """(dx, dw, db) in 64 bits, with bounds."""
    dt = dy.dtype
    dy, x, w = dy.double(), x.double(), w.double()
    dz = dy * slope(z.double(), name) if name != "none" else dy
    # the slope in fp32 (relative to |dy|: it may cancel), and dz's rounding to bf16
    ed = 16 * 2.0 ** -23 * dy.abs() * (1 + (z.double().abs() if z is not None else 0))
    if name in ("none", "relu"):
        ed = 0 * dy
    edz = ed + (eps_out(dt) * dz.abs() if dt == torch.bfloat16 else 0)
    dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
    ex = edz @ w.abs() + eps_sum(w.shape[0], dt) * (dz.abs() @ w.abs())
    ew = edz.T @ x.abs() + eps_sum(x.shape[0], dt) * (dz.abs().T @ x.abs())
    eb = ed.sum(0) + (x.shape[0] + 8) * 2.0 ** -24 * dz.abs().sum(0)
    return (dx, dw, db), (ex, ew, eb)


def xent(x, w, t, b=None, dloss=None):
    """(loss, lse, dx, dw, db) in 64 bits, with bounds.  x rows without a class count as zero
    in dw."""
    dt = x.dtype
    N, Ct = x.shape[0], w.shape[0]
    x, w = x.double(), w.double()
    l = x @ w.T
    mag = x.abs() @ w.abs().T
    if b is not None:
        l = l + b.double()
        mag = mag + torch.where(torch.isfinite(b), b.double().abs(), torch.zeros_like(b.double()))
    lse = torch.logsumexp(l, 1)
    keep = (t >= 0) & (t < Ct)
    tt = torch.where(keep, t, torch.zeros_like(t))
    picked = l.gather(1, tt[:, None])[:, 0]
    loss = torch.where(keep, lse - picked, torch.zeros_like(lse))
    el = (eps_sum(x.shape[1], dt) * mag).max(1).values      # of any logit of the row
    # exp and its sum (2^-22 each term, the terms one after another in up to Ct / 2 steps of a
    # lane would be Ct 2^-24 at worst; they are shared by 16 lanes at least), log, top + log
    elog = el + (8 + Ct / 16) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()
    eloss = torch.where(keep, elog + el + 2.0 ** -23 * (lse.abs() + picked.abs()), torch.zeros_like(el))
    p = torch.exp(l - lse[:, None])
    onehot = torch.zeros_like(p)
    onehot[torch.arange(N, device=x.device), tt] = 1
    valid = int(keep.sum())
    g = dloss.double() if dloss is not None else torch.full((N,), 1.0 / max(1, valid), dtype=torch.float64,
                                                            device=x.device)
    g = torch.where(keep, g, torch.zeros_like(g))
    dl = torch.where(keep[:, None], (p - onehot) * g[:, None], torch.zeros_like(p))
    dl = torch.where(g[:, None] == 0, torch.zeros_like(dl), dl)
    edl = (p * (elog + el + 2.0 ** -21)[:, None] + 2.0 ** -24 * onehot) * g.abs()[:, None]
    edl = torch.where(keep[:, None], edl + 3 * 2.0 ** -24 * dl.abs(), torch.zeros_like(edl))
    er = edl + (eps_out(dt) * dl.abs() if dt == torch.bfloat16 else 0)
    xk = torch.where(keep[:, None], x, torch.zeros_like(x))
    dx, dw, db = dl @ w, dl.T @ xk, dl.sum(0)
    ex = er @ w.abs() + eps_sum(Ct, dt) * (dl.abs() @ w.abs()) + 2.0 ** -23 * dx.abs()
    ew = er.T @ xk.abs() + eps_sum(N, dt) * (dl.abs().T @ xk.abs()) + 2.0 ** -23 * dw.abs()
    eb = edl.sum(0) + (N + 8) * 2.0 ** -24 * dl.abs().sum(0)
    return (loss, lse, dx, dw, db), (eloss, elog, ex, ew, eb)


def orthogonalize(g, steps=5, coeffs=NS, eps=1e-7):
    a, b, c = coeffs
    x = g.double()
    n = torch.linalg.vector_norm(x) + eps
    x = x / n if n > 0 else x
    wide = g.shape[0] <= g.shape[1]
    for _ in range(steps):
        m = x @ x.T if wide else x.T @ x
        m = a * torch.eye(m.shape[0], dtype=torch.float64, device=g.device) + b * m + c * (m @ m)
        x = m @ x if wide else x @ m
    return x
