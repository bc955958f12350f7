"""Plain float64 definitions of the decoder's operators, on the CPU, for the
tests: loops and formulas only, none of the package's code."""
import math

import numpy as np
import torch

F64 = torch.float64
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# smallest step of the type around zero, half of it
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
E32 = 2.0 ** -24


def d64(t):
    return None if t is None else t.detach().cpu().to(F64)


def close(name, got, ref, mag, k=16.0, extra=0.0):
    """|got - ref| within one rounding to got's type and k fp32 roundings of mag,
    the magnitude of the terms that were added up (extra: a bound of its own)."""
    u, tiny = UNIT[got.dtype], TINY[got.dtype]
    g = d64(got)
    tol = u * ref.abs() + tiny + (1 + u) * (k * E32 * mag + extra)
    over = (g - ref).abs() - tol
    over = torch.where(torch.isfinite(ref), over, torch.where((g == ref) | (g.isnan() & ref.isnan()), -1.0, 1.0))
    worst = over.max().item() if over.numel() else -1.0
    at = int(over.argmax()) if over.numel() else 0
    assert worst <= 0.0, (name, "worst element", at, "got", g.flatten()[at].item(), "ref",
                          ref.flatten()[at].item(), "tol", tol.flatten()[at].item())


def layer_norm(x, w, b, eps):
    """y, mean, rstd, and the magnitude of y's terms."""
    d = x.shape[1]
    mean = x.sum(1) / d
    e = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((e * e).sum(1) / d + eps)
    z = e * rstd[:, None]
    y = z if w is None else z * w
    y = y if b is None else y + b
    one = torch.ones(d, dtype=F64)
    mag = (z.abs() + (x.abs().sum(1) / d * rstd)[:, None] + x.abs() * rstd[:, None]) * (one if w is None else w.abs())
    # the variance's relative error grows by what the mean's rounding adds to it
    return y, mean, rstd, mag + (0 if b is None else b.abs())


def layer_norm_bwd(dy, x, mean, rstd, w, add):
    d = x.shape[1]
    z = (x - mean[:, None]) * rstd[:, None]
    zm = (x.abs() + mean.abs()[:, None]) * rstd[:, None]  # magnitude behind z
    v = dy if w is None else dy * w
    c1, c2 = v.sum(1) / d, (v * z).sum(1) / d
    m2 = (v.abs() * zm).sum(1) / d
    dx = rstd[:, None] * (v - c1[:, None] - z * c2[:, None])
    mdx = rstd[:, None] * (v.abs() + (v.abs().sum(1) / d)[:, None] + zm * m2[:, None])
    if add is not None:
        dx, mdx = dx + add, mdx + add.abs()
    return dict(x=(dx, mdx), weight=((dy * z).sum(0), (dy.abs() * zm).sum(0)), bias=(dy.sum(0), dy.abs().sum(0)))


def keep_mask(n, d, p, seed, offset):
    """Philox 4x32-7 in Python integers (small matrices)."""
    M = 0xFFFFFFFF
    thr = math.floor(p * 2 ** 32)
    keep = np.zeros((n, d), bool)
    for r in range(n):
        for q in range((d + 3) // 4):
            c = [q, r, offset & M, offset >> 32]
            k0, k1 = seed & M, seed >> 32
            for _ in range(7):
                a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                c = [(b >> 32) ^ c[1] ^ k0, b & M, (a >> 32) ^ c[3] ^ k1, a & M]
                k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
            for j in range(min(4, d - 4 * q)):
                keep[r, 4 * q + j] = c[j] >= thr
    return torch.from_numpy(keep)


def dropout(x, p, seed, offset, keep=None):
    keep = keep_mask(x.shape[0], x.shape[1], p, seed, offset) if keep is None else keep
    return torch.where(keep, x / (1.0 - p) if p < 1.0 else x, torch.zeros_like(x))


def act(g, name):
    if name == "silu":
        s = torch.special.expit(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    if name == "gelu":
        c = torch.special.ndtr(g)
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    return torch.relu(g), (g > 0).to(F64)
