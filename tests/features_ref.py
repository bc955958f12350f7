"""Plain float64 definitions, on the CPU, of the operators around a decoder's
blocks, for the tests: loops and formulas only, none of the package's code."""
import math

import torch

from decoder_ref import E32, F64


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
