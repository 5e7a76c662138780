"""Plain 64-bit implementations of the operators of a residual block, written from their formulas, on any device."""
import math

import numpy as np
import torch


def fl(t, dtype):
    """Rounded to a type and back to 64 bits."""
    return t.to(dtype).double()


def rms_norm(x, weight, residual, eps):
    """(y, h, rstd): weight (D) or (R, D) or None; h is rounded to the type of x."""
    h = x.double() if residual is None else fl(x.double() + residual.double(), x.dtype)
    rstd = 1.0 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    return h * rstd * _of_rows(weight, x), h, rstd[..., 0]


def _of_rows(weight, x):
    if weight is None:
        return 1.0
    w = weight.double()
    return w if w.dim() == 1 else w.view(w.shape[0], *([1] * (x.dim() - 2)), w.shape[1])


def rms_norm_grad(g, h, rstd, weight, grad_hidden):
    """(dh, dw), and the sums of magnitudes behind dw."""
    n = h.double() * rstd.double()[..., None]
    wg = g.double() * _of_rows(weight, h)
    dh = rstd.double()[..., None] * (wg - n * (wg * n).mean(-1, keepdim=True))
    if grad_hidden is not None:
        dh = dh + grad_hidden.double()
    p = g.double() * n
    D = p.shape[-1]
    p = p.reshape(weight.shape[0], -1, D) if weight is not None and weight.dim() == 2 else p.reshape(1, -1, D)
    dw, size = p.sum(1), p.abs().sum(1)
    return (dh, dw, size) if weight is not None and weight.dim() == 2 else (dh, dw[0], size[0])


def e4m3_values():
    """The magnitudes that 8 bits hold, by their bits."""
    v = []
    for b in range(127):
        e, m = b >> 3, b & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return torch.tensor(v, dtype=torch.float64)


def words(count, worker, seed, round_, layer):
    """Random words of one worker's elements, in Python's integers (slow, apart from any other implementation)."""
    out = []
    for q in range((count + 3) // 4):
        c = [q, worker, round_ & 0xFFFFFFFF, layer << 16 | (round_ >> 32) << 8 | 2]
        k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
        for _ in range(10):
            p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [p1 >> 32 ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, p0 >> 32 ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
            k = [k[0] + 0x9E3779B9 & 0xFFFFFFFF, k[1] + 0xBB67AE85 & 0xFFFFFFFF]
        out += c
    return np.array(out[:count], dtype=np.uint64)


def dropout(x, p, seed, round_, layer, worker, residual, workers):
    parts = list(x) if workers else [x]
    keep = [torch.from_numpy(words(t.numel(), worker + i, seed, round_, layer) >= np.uint64(math.floor(p * 2 ** 32))).view(t.shape)
            for i, t in enumerate(parts)]
    keep = (torch.stack(keep) if workers else keep[0]).to(x.device)
    c = float(np.float32(1.0 / (1.0 - p)))
    y = torch.where(keep, x.double() * c, torch.zeros((), dtype=torch.float64, device=x.device))
    return y if residual is None else y + residual.double()


def activate(z, activation):
    if activation == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if activation == "silu":
        return z / (1 + torch.exp(-z))
    if activation == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z


def slope(z, activation):
    if activation == "relu":
        return (z > 0).double()
    if activation == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p + z * p * (1 - p)
    if activation == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def product(a, b):
    """a b^T in 64 bits, and the sums of magnitudes that bound what rounding can do to it."""
    a, b = a.double(), b.double()
    return a @ b.transpose(-1, -2), a.abs() @ b.abs().transpose(-1, -2)
