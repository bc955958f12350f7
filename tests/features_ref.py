"""Plain float64 definitions, on the CPU, of the operators around a decoder's
blocks, for the tests: loops and formulas only, none of the package's code."""
import math

import torch

from decoder_ref import E32, F64, act as _decoder_act


def embed(table, index, scale):
    y = torch.zeros(len(index), table.shape[1], dtype=F64)
    for i, r in enumerate(index.tolist()):
        if 0 <= r < table.shape[0]:
            y[i] = table[r] * scale
    return y


def embed_bwd(dy, index, m, scale):
    """The table's gradient, and the magnitude of its terms."""
    g, mag = (torch.zeros(m, dy.shape[1], dtype=F64) for _ in range(2))
    keep = (index >= 0) & (index < m)
    g.index_add_(0, index[keep].long(), dy[keep] * scale)
    mag.index_add_(0, index[keep].long(), (dy[keep] * scale).abs())
    return g, mag


def pack8(x):
    """What an 8-bit checkpoint of rows stands for, and its exponents' bytes."""
    n, d = x.shape
    out = torch.full((n, d), math.nan, dtype=F64)
    e = torch.zeros(n, (d + 31) // 32, dtype=torch.uint8)
    for i in range(n):
        for b in range(0, d, 32):
            v = x[i, b:b + 32]
            finite = torch.isfinite(v)
            top = v[finite].abs().max().item() if finite.any() else 0.0
            k = max(math.frexp(top)[1] - 1, -120) if top > 0 else -120
            q = torch.clamp(torch.round(v / 2.0 ** (k - 6)), -127, 127)
            out[i, b:b + 32] = torch.where(finite, q * 2.0 ** (k - 6), math.nan)
            e[i, b // 32] = k + 127
    return out, e


# ------------------------------------------------------ between two blocks

def _stats(v, kind, eps):
    d = v.shape[1]
    mean = v.sum(1) / d if kind == "layer" else torch.zeros(len(v), dtype=F64)
    e = v - mean[:, None]
    return mean, 1.0 / torch.sqrt((e * e).sum(1) / d + eps)


def residual_norm(f, x, post, pre, p, gate, eps):
    """name -> (value, magnitude of the terms behind it: an fp32 evaluation is off by some
    roundings of that)."""
    one, out = torch.ones(f.shape[1], dtype=F64), {}

    def norm(v, mag, k, kind):
        # mag: of v's terms. An error of a mean, or of a variance, reaches the whole row.
        mean, rstd = _stats(v, kind, eps)
        m = mag.sum(1) / v.shape[1]
        out[k + "_rstd"] = (rstd, rstd * (1 + m * rstd) ** 2)
        if kind == "layer":
            out[k + "_mean"] = (mean, m)
        else:
            m = torch.zeros_like(m)
        w, b = p.get(k + "_weight", one), p.get(k + "_bias")
        y = (v - mean[:, None]) * rstd[:, None] * w
        top = (mag + m[:, None]) * rstd[:, None] * (1 + (mag.sum(1) / v.shape[1] * rstd)[:, None]) ** 2 * w.abs()
        return (y, top) if b is None else (y + b, top + b.abs())

    t, mt = (f, f.abs()) if post is None else norm(f, f.abs(), "post", post)
    factor = p.get("scale", one) * (1.0 if gate is None else gate)
    y, my = x + factor * t, x.abs() + factor.abs() * mt
    out["y"] = (y, my)
    if pre is not None:
        out["z"] = norm(y, my, "pre", pre)
    return out


def _norm_bwd(u, mu, v, mean, rstd, kind):
    """Gradient through a norm of v from that of its normalised rows, u; mu: magnitude behind u."""
    d = v.shape[1]
    h = (v - mean[:, None]) * rstd[:, None]
    hm = (v.abs() + mean.abs()[:, None]) * rstd[:, None]
    g = u - h * ((u * h).sum(1) / d)[:, None]
    m = mu + hm * ((mu * hm).sum(1) / d)[:, None]
    if kind == "layer":
        g, m = g - (u.sum(1) / d)[:, None], m + (mu.sum(1) / d)[:, None]
    return g * rstd[:, None], m * rstd[:, None], h, hm


def residual_norm_bwd(dz, dy, f, y, stats, post, pre, p, gate):
    one, zero, out = torch.ones(f.shape[1], dtype=F64), torch.zeros(len(f), dtype=F64), {}
    g = torch.zeros_like(f) if dy is None else dy
    mg = g.abs()
    stat = lambda k: stats[k] if stats.get(k) is not None else zero
    if pre is not None:
        u = dz * p.get("pre_weight", one)
        add, m, h, hm = _norm_bwd(u, u.abs(), y, stat("pre_mean"), stats["pre_rstd"], pre)
        g, mg = g + add, mg + m
        out["pre_weight"], out["pre_bias"] = ((dz * h).sum(0), (dz.abs() * hm).sum(0)), (dz.sum(0), dz.abs().sum(0))
    out["x"] = (g, mg)
    s, w, b = p.get("scale", one), p.get("post_weight", one), p.get("post_bias", 0 * one)
    k = torch.ones_like(f) if gate is None else gate.expand_as(f)
    dt, mdt = g * k * s, mg * (k * s).abs()
    if post is None:
        h, hm = f, f.abs()
        out["f"] = (dt, mdt)
    else:
        df, m, h, hm = _norm_bwd(dt * w, mdt * w.abs(), f, stat("post_mean"), stats["post_rstd"], post)
        out["f"] = (df, m)
        out["post_weight"], out["post_bias"] = ((dt * h).sum(0), (mdt * hm).sum(0)), (dt.sum(0), mdt.sum(0))
    t, mt = h * w + b, hm * w.abs() + b.abs()
    out["scale"] = ((g * k * t).sum(0), (mg * k.abs() * mt).sum(0))
    by, mby = g * s * t, mg * s.abs() * mt
    out["gate"] = (by, mby) if gate is None or gate.shape == f.shape else (by.sum(1, keepdim=True), mby.sum(1, keepdim=True))
    return out


# ------------------------------------------------------------ linear layer

def act(z, name):
    """An activation, its derivative, and a bound of the second one's size."""
    if name is None:
        return z, torch.ones_like(z), 0.0
    if name == "sigmoid":
        s = torch.special.expit(z)
        return s, s * torch.special.expit(-z), 0.1
    a, da = _decoder_act(z, name)
    return a, da, dict(silu=0.5, gelu=0.8, relu=0.0)[name]


def linear(x, w, b, name, res):
    """y and the magnitude behind it."""
    z, mz = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        z, mz = z + b, mz + b.abs()
    a, da, _ = act(z, name)
    m = mz if name is None else 1.1 * mz + a.abs()  # no act here has a slope above 1.13
    return (a, m) if res is None else (a + res, m + res.abs())


def linear_bwd(dy, x, w, b, name, u, kept):
    """name -> (value, magnitude of the fp32 sums' terms, standard deviation that rounding
    dz to unit u, and the slopes to `kept` (0: not kept), leaves, to first order)."""
    z, mz = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        z, mz = z + b, mz + b.abs()
    _, da, bend = act(z, name)
    dz = dy * da
    sdz = torch.zeros_like(dz)
    if name is not None:
        sdz = u * dz.abs() + kept * (dz.abs() + 2.0 ** -8 * dy.abs()) + 16 * E32 * dy.abs() * (da.abs() + bend * mz)
    if name == "relu":  # its slope jumps where the fp32 sum may have either sign
        sdz = sdz + torch.where(z.abs() <= 16 * E32 * mz, dy.abs(), torch.zeros_like(z))
    return dict(x=(dz @ w, dz.abs() @ w.abs(), (sdz ** 2 @ w ** 2).sqrt()),
                w=(dz.T @ x, dz.abs().T @ x.abs(), ((sdz ** 2).T @ x ** 2).sqrt()),
                b=(dz.sum(0), dz.abs().sum(0), (sdz ** 2).sum(0).sqrt()))
