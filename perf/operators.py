"""The operators of a per-Gaussian decoder, as they are timed and checked.

A decoder turns learned features (one row per Gaussian, or per token of a
feed-forward reconstruction) into attributes. Its block is
x + dropout(ffn(layer_norm(x))), and a case is one operator of it:

  norm      layer norm of n rows of width d: y, and the rows' mean and 1/sd
  norm_bwd  its gradients dx (added to a gradient that comes by the residual
            path), dweight, dbias
  drop      residual + dropout(x), the mask from a counter-based generator
  drop_bwd  dropout's gradient, the mask made again
  ffn       the gated feed-forward block y = residual + dropout(h Wd' + bd),
            h = act(x Wg' + bg) * (x Wu' + bu)
  ffn_step  its forward and backward pass together, as a training step has
            them: y and the gradients of x and of every weight and bias

The generator is Philox 4x32 with 7 rounds (Salmon et al., "Parallel random
numbers: as easy as 1, 2, 3", 2011): element (row, col) takes word col % 4 of
the block of counter (col // 4, row, offset low, offset high) under the key
(seed low, seed high), and is kept if that word is at least p 2^32.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ITEM = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
# rows that the plain form and the 64-bit one work on at a time where they make
# several temporaries as large as their input
CHUNK = 1 << 17


def listed():
    return [
        # one query's features before its block: latency
        dict(name="norm_one_row", what="norm", dtype="bf16", n=1, d=2048),
        # every Gaussian's features of the 1M-Gaussian block
        dict(name="norm_1m_x64", what="norm", dtype="bf16", n=1000000, d=64),
        # the same features on the way back, in the parameters' own 32 bits
        dict(name="norm_bwd_1m_x64", what="norm_bwd", dtype="f32", n=1000000, d=64),
        # wide tokens; and a ragged batch of an odd width
        dict(name="norm_bwd_16k_x4096", what="norm_bwd", dtype="bf16", n=16384, d=4096),
        dict(name="norm_bwd_odd", what="norm_bwd", dtype="f16", n=4099, d=1001),
        # the residual path over every Gaussian
        dict(name="drop_1m_x64", what="drop", dtype="bf16", n=1000000, d=64, p=0.1),
        # all attributes (SH 3: 59 floats) of a small block: latency, an odd width
        dict(name="drop_bwd_3001_x59", what="drop_bwd", dtype="f32", n=3001, d=59, p=0.25),
        # one new token through a wide block: the weights are read once
        dict(name="ffn_one_row", what="ffn", dtype="bf16", act="silu", n=1, d=2048, h=5632, o=2048, p=0.0, bias=False),
        # a ragged batch of tokens, no size a multiple of a tile
        dict(name="ffn_odd", what="ffn", dtype="f16", act="gelu", n=5003, d=1000, h=2731, o=1000, p=0.1, bias=True),
        # the decoder's block for every Gaussian, one training step
        dict(name="ffn_step_1m_x64", what="ffn_step", dtype="bf16", act="silu", n=1000000, d=64, h=128, o=64, p=0.1, bias=True),
        # wide tokens, one training step: matrix products bound it
        dict(name="ffn_step_8k_x2048", what="ffn_step", dtype="bf16", act="silu", n=8192, d=2048, h=5632, o=2048, p=0.1, bias=False),
        # a decoder of the 59 attributes in 32 bits, for the ring scene's Gaussians
        dict(name="ffn_step_f32", what="ffn_step", dtype="f32", act="gelu", n=65536, d=96, h=256, o=59, p=0.0, bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        k = _kind(c)
        top[k] = tuple(max(a, b) for a, b in zip(top.get(k, (0, 0)), (w["bytes"], w["flops"])))
    while True:
        what = rng.choice(["norm", "norm_bwd", "drop", "drop_bwd", "ffn", "ffn", "ffn_step", "ffn_step"])
        c = dict(what=what, dtype=rng.choice(["bf16", "f16", "f32"]))
        if what.startswith("ffn"):
            c["act"] = rng.choice(["silu", "gelu"])
            c["bias"] = rng.random() < 0.5
            c["p"] = rng.choice([0.0, 0.1, 0.5])
            shape = rng.choice(["few", "points", "tokens"])
            if shape == "few":  # single tokens and small batches of them
                c["n"] = _log_int(rng, 1, 64)
                c["d"], c["h"] = _log_int(rng, 64, 2048), _log_int(rng, 128, 5632)
            elif shape == "points":  # one row per Gaussian
                c["n"] = _log_int(rng, 1000, 1000000)
                c["d"], c["h"] = _log_int(rng, 16, 256), _log_int(rng, 16, 512)
            else:
                c["n"] = _log_int(rng, 65, 8192)
                c["d"], c["h"] = _log_int(rng, 256, 2048), _log_int(rng, 256, 5632)
            c["o"] = c["d"]
            if rng.random() < 0.6:  # most widths are multiples of 8
                c["d"], c["h"], c["o"] = (max(16, (v + 4) // 8 * 8) for v in (c["d"], c["h"], c["o"]))
            if rng.random() < 0.25:
                c["o"] = rng.randint(16, 64)
        else:
            c["n"], c["d"] = _log_int(rng, 1, 1000000), _log_int(rng, 16, 4096)
            if rng.random() < 0.6:
                c["d"] = max(16, (c["d"] + 4) // 8 * 8)
            if what.startswith("drop"):
                c["p"] = rng.choice([0.1, 0.25, 0.5])
        w = work(c)
        b, f = top[_kind(c)]
        if w["bytes"] <= b and w["flops"] <= f:
            return c


def _kind(c):
    return c["what"].split("_")[0]


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    n, d = case["n"], case["d"]

    def randn(*shape, scale=1.0, shift=0.0):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)
        return x.mul_(scale).add_(shift).to(t)

    s = dict(case)
    # what the generator takes: a run's seed, and a number for each call
    s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), seed * 1000003 % (1 << 40) + 7
    what = case["what"]
    if what in ("norm", "norm_bwd"):
        # features drift apart in mean and scale by channel as a model learns
        x = torch.randn(n, d, generator=g, device="cuda", dtype=torch.float32)
        x *= 0.5 + torch.rand(d, generator=g, device="cuda")
        x += 0.3 * torch.randn(d, generator=g, device="cuda")
        s["x"] = x.to(t)
        s["weight"], s["bias"] = randn(d, scale=0.2, shift=1.0), randn(d, scale=0.1)
        if what == "norm_bwd":
            # the forward's statistics, which a training step keeps
            mean, var = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            for i in range(0, n, CHUNK):
                v = s["x"][i:i + CHUNK].float()
                mean[i:i + CHUNK] = v.mean(1)
                var[i:i + CHUNK] = (v - mean[i:i + CHUNK, None]).square().mean(1)
            s["mean"], s["rstd"] = mean, torch.rsqrt(var + EPS)
            s["dy"] = randn(n, d)
            s["add"] = randn(n, d)
    elif what in ("drop", "drop_bwd"):
        s["x"] = randn(n, d)
        if what == "drop":
            s["residual"] = randn(n, d)
    else:
        h, o = case["h"], case["o"]
        s["x"] = randn(n, d)
        w = dict(w_gate=randn(h, d, scale=d ** -0.5), w_up=randn(h, d, scale=d ** -0.5),
                 w_down=randn(o, h, scale=h ** -0.5))
        if case["bias"]:
            w.update(b_gate=randn(h, scale=0.1), b_up=randn(h, scale=0.1), b_down=randn(o, scale=0.1))
        s["w"] = w
        # a block that changes the width (the last one, to the attributes) has no residual path
        s["residual"] = s["x"] if o == d else None
        if what == "ffn_step":
            s["dy"] = randn(n, o)
    return s


# --------------------------------------------------------------- plain form

def _words(n, d, seed, offset, row0, device):
    """Philox 4x32-7 in 64-bit integers: the words of rows row0.. of width d."""
    m = 0xFFFFFFFF
    cols = (d + 3) // 4
    c0 = torch.arange(cols, dtype=torch.int64, device=device).expand(n, cols)
    c1 = torch.arange(row0, row0 + n, dtype=torch.int64, device=device)[:, None].expand(n, cols)
    c2 = torch.full_like(c0, offset & m)
    c3 = torch.full_like(c0, offset >> 32 & m)
    k0, k1 = seed & m, seed >> 32 & m
    for _ in range(7):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # exact modulo 2^64
        c0, c1, c2, c3 = (p1 >> 32 & m) ^ c1 ^ k0, p1 & m, (p0 >> 32 & m) ^ c3 ^ k1, p0 & m
        k0, k1 = k0 + 0x9E3779B9 & m, k1 + 0xBB67AE85 & m
    return torch.stack((c0, c1, c2, c3), 2).reshape(n, 4 * cols)[:, :d]


def _dropout(x, p, seed, offset, row0=0):
    """Dropout of fp32 rows row0.. of a matrix."""
    if p == 0.0:
        return x
    keep = _words(x.shape[0], x.shape[1], seed, offset, row0, x.device) >= int(p * 2.0 ** 32)
    return torch.where(keep, x * (1.0 / (1.0 - p)), torch.zeros_like(x))


def _dropout_chunks(x, s, residual=None):
    t = x.dtype
    out = torch.empty_like(x)
    for i in range(0, x.shape[0], CHUNK):
        y = _dropout(x[i:i + CHUNK].float(), s["p"], s["seed"], s["offset"], i)
        if residual is not None:
            y = residual[i:i + CHUNK].float() + y
        out[i:i + CHUNK] = y.to(t)
    return out


def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        e = 1.0 / (1.0 + torch.exp(-g))
        return g * e, e * (1.0 + g * (1.0 - e))
    c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = torch.rsqrt(x.square().mean(1) + EPS)
    y = x * rstd[:, None] * s["weight"].float() + s["bias"].float()
    return dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)


def _plain_norm_bwd(s):
    t = s["x"].dtype
    dy = s["dy"].float()
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dw, db = (dy * xh).sum(0), dy.sum(0)
    dyw = dy * s["weight"].float()
    dx = dyw - dyw.mean(1, keepdim=True) - xh * (dyw * xh).mean(1, keepdim=True)
    dx = dx * s["rstd"][:, None] + s["add"].float()
    return dict(dx=dx.to(t), dweight=dw.to(t), dbias=db.to(t))


def _plain_ffn(s):
    t = s["x"].dtype
    w = {k: v.float() for k, v in s["w"].items()}
    x = s["x"].float()
    g, u = x @ w["w_gate"].t(), x @ w["w_up"].t()
    if s["bias"]:
        g, u = g + w["b_gate"], u + w["b_up"]
    a, da = _act(g, s["act"])
    hid = a * u
    y = hid @ w["w_down"].t()
    if s["bias"]:
        y = y + w["b_down"]
    for i in range(0, y.shape[0], CHUNK):
        y[i:i + CHUNK] = _dropout(y[i:i + CHUNK], s["p"], s["seed"], s["offset"], i)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(y=y.to(t))
    if s["what"] == "ffn":
        return out
    dz = s["dy"].float()
    if s["p"] > 0.0:
        dz = dz.clone()
        for i in range(0, dz.shape[0], CHUNK):
            dz[i:i + CHUNK] = _dropout(dz[i:i + CHUNK], s["p"], s["seed"], s["offset"], i)
    dh = dz @ w["w_down"]
    dg, du = dh * u * da, dh * a
    out["x"] = (dg @ w["w_gate"] + du @ w["w_up"]).to(t)
    out["w_gate"], out["w_up"] = (dg.t() @ x).to(t), (du.t() @ x).to(t)
    out["w_down"] = (dz.t() @ hid).to(t)
    if s["bias"]:
        out["b_gate"], out["b_up"], out["b_down"] = dg.sum(0).to(t), du.sum(0).to(t), dz.sum(0).to(t)
    return out


def run(s):
    what = s["what"]
    if own:
        return _own(s)
    if what == "norm":
        return _plain_norm(s)
    if what == "norm_bwd":
        return _plain_norm_bwd(s)
    if what == "drop":
        return _dropout_chunks(s["x"], s, s["residual"])
    if what == "drop_bwd":
        return _dropout_chunks(s["x"], s)
    return _plain_ffn(s)


def _own(s):
    from paper_2608_27735_amd import api

    what = s["what"]
    if what == "norm":
        return api.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    if what == "norm_bwd":
        r = api.layer_norm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], add=s["add"])
        return dict(dx=r["x"], dweight=r["weight"], dbias=r["bias"])
    drop = dict(p=s["p"], seed=s["seed"], offset=s["offset"])
    if what == "drop":
        return api.dropout(s["x"], residual=s["residual"], **drop)
    if what == "drop_bwd":
        return api.dropout_bwd(s["x"], **drop)
    train = what == "ffn_step"
    r = api.gated_ffn(s["x"], s["w"], act=s["act"], residual=s["residual"], save=train, **drop)
    out = dict(y=r["y"])
    if train:
        out.update(api.gated_ffn_bwd(s["dy"], s["x"], s["w"], act=s["act"], saved=r["saved"], **drop))
    return out


# -------------------------------------------------------------------- work

def work(case):
    n, d, b = case["n"], case["d"], ITEM[case["dtype"]]
    what = case["what"]
    if what == "norm":
        return {"bytes": b * (2 * n * d + 2 * d) + 8 * n, "flops": 8 * n * d}
    if what == "norm_bwd":
        return {"bytes": b * (4 * n * d + 3 * d) + 8 * n, "flops": 14 * n * d}
    if what == "drop":
        return {"bytes": b * 3 * n * d, "flops": 2 * n * d}
    if what == "drop_bwd":
        return {"bytes": b * 2 * n * d, "flops": n * d}
    h, o = case["h"], case["o"]
    weights = 2 * h * d + o * h + ((2 * h + o) if case["bias"] else 0)
    if what == "ffn":
        return {"bytes": b * (n * (d + o) + weights), "flops": 2 * n * h * (2 * d + o)}
    return {"bytes": b * (n * (2 * d + 2 * o) + 2 * weights), "flops": 3 * 2 * n * h * (2 * d + o)}


# ----------------------------------------------------------- 64-bit values

def _kept64(row0, n, d, p, seed, offset):
    """Truth values of the kept elements, in unsigned 64-bit integers."""
    quads = -(-d // 4)
    u32 = np.uint64(0xFFFFFFFF)
    s32 = np.uint64(32)
    x = [np.broadcast_to(np.arange(quads, dtype=np.uint64), (n, quads)),
         np.broadcast_to(np.arange(row0, row0 + n, dtype=np.uint64)[:, None], (n, quads)),
         np.uint64(offset % (1 << 32)), np.uint64(offset // (1 << 32) % (1 << 32))]
    for r in range(7):
        key = [(seed + r * 0x9E3779B9) % (1 << 32), (seed // (1 << 32) + r * 0xBB67AE85) % (1 << 32)]
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> s32) ^ x[1] ^ np.uint64(key[0]), b & u32, (a >> s32) ^ x[3] ^ np.uint64(key[1]), a & u32]
    thr = np.uint64(math.floor(p * 4294967296.0))
    keep = np.empty((n, quads, 4), dtype=bool)
    for j in range(4):
        keep[:, :, j] = x[j] >= thr
    return keep.reshape(n, 4 * quads)[:, :d]


def _drop64(v, s):
    """Dropout of a 64-bit matrix on the GPU, in place."""
    if s["p"] > 0.0:
        for i in range(0, v.shape[0], CHUNK):
            part = v[i:i + CHUNK]
            keep = torch.from_numpy(np.ascontiguousarray(
                _kept64(i, part.shape[0], part.shape[1], s["p"], s["seed"], s["offset"]))).to(v.device)
            part.div_(1.0 - s["p"]).masked_fill_(~keep, 0.0)
    return v


def _sigmoid64(g):
    return torch.special.expit(g)


def _normal_cdf64(g):
    return torch.special.ndtr(g)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    what = case["what"]
    if what == "norm":
        x = s["x"].to(f64)
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        y = torch.addcmul(s["bias"].to(f64), (x - mean) / torch.sqrt(var + EPS), s["weight"].to(f64))
        return dict(y=y, mean=mean[:, 0], rstd=1.0 / torch.sqrt(var[:, 0] + EPS))
    if what == "norm_bwd":
        # with z the standardised row and v = dy * weight: dx = (v - (v.1) / d - z (v.z) / d) / sd
        z = (s["x"].to(f64) - s["mean"].to(f64)[:, None]) * s["rstd"].to(f64)[:, None]
        dy = s["dy"].to(f64)
        dw, db = torch.linalg.vecdot(dy, z, dim=0), torch.sum(dy, 0)
        v = dy * s["weight"].to(f64)
        along = torch.linalg.vecdot(v, z, dim=1)[:, None] / case["d"]
        across = torch.sum(v, 1, keepdim=True) / case["d"]
        dx = s["add"].to(f64) + s["rstd"].to(f64)[:, None] * (v - across - z * along)
        return dict(dx=dx, dweight=dw, dbias=db)
    if what in ("drop", "drop_bwd"):
        v = _drop64(s["x"].to(f64), s)
        return v + s["residual"].to(f64) if what == "drop" else v
    w = {k: v.to(f64) for k, v in s["w"].items()}
    n, d, h, o = case["n"], case["d"], case["h"], case["o"]
    zero = lambda m: torch.zeros(m, dtype=f64, device="cuda")
    bg, bu, bd = w.get("b_gate", zero(h)), w.get("b_up", zero(h)), w.get("b_down", zero(o))
    x = s["x"].to(f64)
    g, u = torch.addmm(bg, x, w["w_gate"].T), torch.addmm(bu, x, w["w_up"].T)
    if case["act"] == "silu":
        q = _sigmoid64(g)
        a, slope = g * q, q + g * q * (1.0 - q)
    else:
        q = _normal_cdf64(g)
        a, slope = g * q, q + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
    y = _drop64(torch.addmm(bd, a * u, w["w_down"].T), s)
    if s["residual"] is not None:
        y += s["residual"].to(f64)
    out = dict(y=y)
    if what == "ffn":
        return out
    dz = _drop64(s["dy"].to(f64), s)
    dh = torch.mm(dz, w["w_down"])
    out["w_down"] = torch.mm(dz.T, a * u)
    dg, du = dh * u * slope, dh * a
    del dh, g, u, a, slope
    out["w_gate"], out["w_up"] = torch.mm(dg.T, x), torch.mm(du.T, x)
    out["x"] = torch.addmm(torch.mm(dg, w["w_gate"]), du, w["w_up"])
    if case["bias"]:
        out["b_gate"], out["b_up"], out["b_down"] = dg.sum(0), du.sum(0), dz.sum(0)
    return out
