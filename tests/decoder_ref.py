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
    """Philox 4x32-7, its words as unsigned 64-bit integers."""
    M, S = np.uint64(0xFFFFFFFF), np.uint64(32)
    quads = (d + 3) // 4
    c = [np.tile(np.arange(quads, dtype=np.uint64), (n, 1)),
         np.repeat(np.arange(n, dtype=np.uint64)[:, None], quads, 1),
         np.full((n, quads), offset & 0xFFFFFFFF, np.uint64), np.full((n, quads), offset >> 32, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> S) ^ c[1] ^ np.uint64(k0), b & M, (a >> S) ^ c[3] ^ np.uint64(k1), a & M]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    keep = np.stack(c, 2).reshape(n, 4 * quads)[:, :d] >= np.uint64(math.floor(p * 2 ** 32))
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


def ffn(x, w, name, u, res=None, keep=None, p=0.0, dy=None):
    """The gated feed-forward block and its gradients: name -> (value, magnitude
    of the fp32 sums' terms, standard deviation that rounding the stored
    intermediates to unit u leaves, to first order)."""
    z = lambda k, n: w[k] if w.get(k) is not None else torch.zeros(n, dtype=F64)
    h, o = w["w_gate"].shape[0], w["w_down"].shape[0]
    g, up = x @ w["w_gate"].T + z("b_gate", h), x @ w["w_up"].T + z("b_up", h)
    mg = x.abs() @ w["w_gate"].abs().T + z("b_gate", h).abs()
    mu = x.abs() @ w["w_up"].abs().T + z("b_up", h).abs()
    a, da = act(g, name)
    hid = a * up
    # fp32 sums reach h too
    sh = u * hid.abs() + 8 * E32 * (da.abs() * mg * up.abs() + a.abs() * mu + hid.abs())
    y = hid @ w["w_down"].T + z("b_down", o)
    my = hid.abs() @ w["w_down"].abs().T + z("b_down", o).abs()
    sy = (sh ** 2 @ w["w_down"].T ** 2).sqrt()
    keep = torch.ones_like(y, dtype=torch.bool) if keep is None else keep
    scale = 1.0 / (1.0 - p) if p < 1.0 else 0.0
    y, my, sy = (torch.where(keep, v * scale, torch.zeros_like(v)) for v in (y, my, sy))
    if res is not None:
        y, my = y + res, my + res.abs()
    out = dict(y=(y, my, sy))
    if dy is None:
        return out
    dz = torch.where(keep, dy * scale, torch.zeros_like(dy))
    sdz = u * dz.abs() if p > 0 else torch.zeros_like(dz)
    dh = dz @ w["w_down"]
    sdh = (sdz ** 2 @ w["w_down"] ** 2).sqrt() + 8 * E32 * (dz.abs() @ w["w_down"].abs())
    dg, du = dh * up * da, dh * a
    sdg = u * (dg.abs() * 2 + (dh * up * g).abs()) + (up * da).abs() * sdh + \
        8 * E32 * ((dh * da).abs() * mu + (dh * up).abs() * mg)
    if name == "relu":  # its derivative jumps where the fp32 sum may have either sign
        sdg = sdg + torch.where(g.abs() <= 16 * E32 * mg, (dh * up).abs(), torch.zeros_like(g))
    sdu = u * (du.abs() + (dh * da * g).abs()) + a.abs() * sdh + 8 * E32 * dh.abs() * mg * da.abs()
    both = lambda f: f(dg, sdg, "w_gate") + f(du, sdu, "w_up")
    out["x"] = (both(lambda v, s, k: v @ w[k]), both(lambda v, s, k: v.abs() @ w[k].abs()),
                both(lambda v, s, k: s ** 2 @ w[k] ** 2).sqrt())
    for k, v, s in (("w_gate", dg, sdg), ("w_up", du, sdu)):
        out[k] = (v.T @ x, v.abs().T @ x.abs(), ((s ** 2).T @ x ** 2).sqrt())
    out["w_down"] = (dz.T @ hid, dz.abs().T @ hid.abs(),
                     ((sdz ** 2).T @ hid ** 2 + (dz ** 2).T @ sh ** 2).sqrt())
    for k, v, s in (("b_gate", dg, sdg), ("b_up", du, sdu), ("b_down", dz, sdz)):
        out[k] = (v.sum(0), v.abs().sum(0), (s ** 2).sum(0).sqrt())
    return out
