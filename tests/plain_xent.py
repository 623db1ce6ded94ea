"""Softmax cross entropy in 64 bits with bounds in which a class that is masked (p = 0) has no part,
and which hardly grow with the number of classes.

Of a row with logits l_c, each computed within e_c (plain_finetune.eps_sum's sum of K products, and
the bias' rounding): lse = log sum exp l_c moves by at most max e_c over the classes with p_c > 0.  The
sum itself: exp by 2^x of (l - top) log2 e, relative error 2^-22 and 3 * 2^-24 |l - top| (the
difference, log2 e and the product round), which weighted by p_c is at most 3 * 2^-24 (1 + log Ct) in
all; a term takes part in up to 8 x 9 additions and rescalings of its tile's half, or Ct / 256 of its
thread, and 150 more of lanes, warps and tiles, 2^-24 each of a sum of positive terms.  Then log and
top + log, 2^-23 each of their result.
"""
import math

import torch

from plain_finetune import eps_out, eps_sum


def xent(x, w, t, b=None, dloss=None):
    """(loss, lse, dx, dw, db) in 64 bits, with bounds; rows without a class count as zero."""
    dt, (N, K), Ct = x.dtype, x.shape, w.shape[0]
    x, w = x.double(), w.double()
    l, mag = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        b = b.double()
        l = l + b
        mag = mag + torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b))
    lse = torch.logsumexp(l, 1)
    keep = (t >= 0) & (t < Ct)
    tt = torch.where(keep, t, torch.zeros_like(t))[:, None]
    picked = l.gather(1, tt)[:, 0]
    zero = torch.zeros_like(lse)
    loss = torch.where(keep, lse - picked, zero)
    p = torch.exp(l - lse[:, None])
    ec = eps_sum(K, dt) * torch.where(p > 0, mag, torch.zeros_like(mag))
    el = ec.max(1).values
    elog = el + (230 + Ct / 256) * 2.0 ** -24 + 2.0 ** -22 * (2 + math.log(Ct)) + 2.0 ** -23 * lse.abs()
    et = eps_sum(K, dt) * mag.gather(1, tt)[:, 0]
    eloss = torch.where(keep, elog + et + 2.0 ** -23 * (lse.abs() + picked.abs()), zero)
    valid = int(keep.sum())
    g = dloss.double() if dloss is not None else torch.full_like(lse, 1.0 / max(1, valid))
    g = torch.where(keep, g, zero)
    far = torch.where(p > 0, (l - lse[:, None]).abs(), torch.zeros_like(p))
    edl = p * (elog[:, None] + ec + 2.0 ** -21 * (1 + far))
    edl.scatter_add_(1, tt, torch.full_like(lse, 2.0 ** -24)[:, None])
    dl = p.scatter_add(1, tt, -torch.ones_like(lse)[:, None]) * g[:, None]
    dl = torch.where(keep[:, None], dl, torch.zeros_like(dl))
    edl = torch.where(keep[:, None], edl * g.abs()[:, None] + 3 * 2.0 ** -24 * dl.abs(), torch.zeros_like(edl))
    er = edl + (eps_out(dt) * dl.abs() if dt == torch.bfloat16 else 0)
    xk = torch.where(keep[:, None], x, torch.zeros_like(x))
    dx, dw, db = dl @ w, dl.T @ xk, dl.sum(0)
    ex = er @ w.abs() + eps_sum(Ct, dt) * (dl.abs() @ w.abs()) + 2.0 ** -23 * dx.abs()
    ew = er.T @ xk.abs() + eps_sum(N, dt) * (dl.abs().T @ xk.abs()) + 2.0 ** -23 * dw.abs()
    eb = edl.sum(0) + (N + 8) * 2.0 ** -24 * dl.abs().sum(0)
    return (loss, lse, dx, dw, db), (eloss, elog, ex, ew, eb)
