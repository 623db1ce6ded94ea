"""Plain forms of dropout, of the quantizing of rows and of a dense layer in 8-bit integers (torch,
any device), and bounds on what fp32 arithmetic and roundings to fp32 or bf16 may differ from them by.

Words and codes are whole numbers, defined step by step: they have to be equal.
Dropout.  1 / (1 - p) rounded to fp32 (2^-24 of it), a product (2^-24), a sum (2^-24), a rounding to
the result's type: (2 2^-24) |x / (1 - p)| + 2^-24 |y|, then 2^-p |y|.
Dense layer.  A sum of products of codes is an exact integer, rounded to fp32 once (2^-24, nothing
below 2^24).  Two products with scales (2 2^-24), the bias (2^-24 of z), then as dense_forward:
|act'| <= 1.13, erf and exp good to 8 2^-23 |z|, the residual's addition 2^-24 |y|, the rounding.
"""
import torch

from plain_finetune import act as activation

LOW = 0xFFFFFFFF


def philox(block, offset, seed):
    """The four words of a counter, in Python's integers."""
    c, k = [block & LOW, block >> 32, offset & LOW, offset >> 32], [seed & LOW, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return c


def words(n, offset, seed, first=0, device="cpu"):
    """The words of elements first (a multiple of 4) to first + n - 1, int64."""
    i = first // 4 + torch.arange((n + 3) // 4, device=device)
    c = [i & LOW, i >> 32, torch.full_like(i, offset & LOW), torch.full_like(i, offset >> 32)]
    k = [seed & LOW, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # (the low 64 bits)
        c = [(b >> 32 & LOW) ^ c[1] ^ k[0], b & LOW, (a >> 32 & LOW) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return torch.stack(c, 1).flatten()[:n]


def kept(shape, p, offset, seed, device="cpu"):
    n = shape[0] * shape[1]
    return (words(n, offset, seed, device=device) >= min(round(p * 2 ** 32), LOW)).view(shape)


def dropout(x, p, offset, seed, r=None):
    """(y in 64 bits, bound before the rounding to a type)."""
    keep = kept(x.shape, p, offset, seed, x.device)
    y = torch.where(keep, x.double() / (1 - p), torch.zeros((), dtype=torch.float64, device=x.device))
    e = 2 * 2.0 ** -24 * y.abs()
    if r is not None:
        y = y + r.double()
        e = e + 2.0 ** -24 * y.abs()
    return y, e


def quantize(x):
    """(codes int8, scale float32) in the steps of the definition, on the host."""
    x = x.float().cpu()
    top = x.abs().amax(1)
    s = torch.maximum(top * torch.tensor(1 / 127, dtype=torch.float32), torch.tensor(2.0 ** -126))
    s = torch.where(torch.isnan(top), top, s)
    finite = torch.isfinite(top)[:, None]
    q = torch.round(torch.where(finite, x, torch.zeros(())) * torch.reciprocal(s)[:, None])
    return torch.where(finite, q, torch.zeros(())).clamp(-127, 127).to(torch.int8), s


def dense(q, xs, w, ws, b=None, name="none", r=None):
    """(y in 64 bits, bound before the rounding) of codes q [N, Cs], w [Ct, Cs] with their scales."""
    qd, wd = q.double(), w.double()
    scale = xs.double()[:, None] * ws.double()
    z = (qd @ wd.T) * scale
    ez = 3 * 2.0 ** -24 * z.abs()
    if b is not None:
        z = z + b.double()
        ez = ez + 2.0 ** -24 * z.abs()
    y = activation(z, name)
    ey = 1.13 * ez + (8 * 2.0 ** -23 * z.abs() if name in ("gelu", "silu") else 0)
    if r is not None:
        y = y + r.double()
        ey = ey + 2.0 ** -24 * y.abs()
    return y, ey
