"""Layer norm and dropout of the decoder against float64 definitions, at the
widths, strides and values where they can go wrong. Tolerances: one rounding to
the output's type and a few fp32 roundings of the magnitude of the terms."""
import math

import pytest
import torch

import decoder_ref as R

pytestmark = pytest.mark.gpu

DT = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]


def say(*a):
    print("[case]", *a, flush=True)


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_27735_amd import api
    return api


def rand(seed, n, d, dtype, pad=0, skip=0, scale=1.0, shift=0.0):
    """An n x d matrix on the GPU, `pad` elements between its rows, `skip`
    elements into its allocation."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, d, generator=g) * scale + shift).to(dtype)
    buf = torch.full((skip + n * (d + pad),), float("nan"), dtype=dtype, device="cuda")
    v = buf[skip:].view(n, d + pad)[:, :d]
    v.copy_(x)
    return v


# every row shape of the kernels (8 to 64 lanes, a wave with two vectors, a
# workgroup with one to four, rows read again), odd widths, one element
WIDTHS = [1, 2, 7, 16, 59, 64, 100, 129, 255, 256, 500, 1001, 1024, 2048, 2053, 4096, 8192, 8200, 20001]


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_both_ways(api, dtype, d):
    n = 37 if d < 2000 else 5
    for pad, skip, wtype, eps in ((0, 0, dtype, 1e-5), (3, 1, torch.float32, 1e-3)):
        say("layer_norm", dtype, n, d, pad, skip, wtype)
        x = rand(1, n, d, dtype, pad, skip, scale=2.0, shift=0.5)
        w, b = rand(2, 1, d, wtype, scale=0.3, shift=1.0)[0], rand(3, 1, d, wtype)[0]
        dy, add = rand(4, n, d, dtype, 2 * pad, skip), rand(5, n, d, dtype, pad)
        for ww, bb in ((w, b), (None, None)):
            f = api.layer_norm(x, ww, bb, eps=eps)
            y, mean, rstd, mag = R.layer_norm(R.d64(x), R.d64(ww), R.d64(bb), eps)
            xm = R.d64(x).abs().mean(1)
            R.close("mean", f["mean"], mean, xm)
            # of a relative error e of the variance, e / 2 reaches rstd
            R.close("rstd", f["rstd"], rstd, rstd * (1 + xm * rstd) ** 2)
            R.close("y", f["y"], y, mag * (1 + (xm * rstd)[:, None]) ** 2)
            for aa in (add, None):
                g = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], ww, add=aa,
                                       wdtype=None if ww is not None else wtype)
                ref = R.layer_norm_bwd(R.d64(dy), R.d64(x), R.d64(f["mean"]), R.d64(f["rstd"]), R.d64(ww), R.d64(aa))
                for k in ("x", "weight", "bias"):
                    R.close("d" + k, g[k], *ref[k])
                assert g["weight"].dtype == (wtype if ww is None else ww.dtype)


@pytest.mark.parametrize("n", [0, 1, 2, 3, 63, 1023, 1025, 40000])
def test_layer_norm_row_counts(api, n):
    d = 72
    say("rows", n)
    x, dy = rand(1, n, d, torch.float32), rand(2, n, d, torch.float32)
    w, b = rand(3, 1, d, torch.float32)[0], rand(4, 1, d, torch.float32)[0]
    f = api.layer_norm(x, w, b)
    y, mean, rstd, mag = R.layer_norm(R.d64(x), R.d64(w), R.d64(b), 1e-5)
    R.close("y", f["y"], y, 4 * mag)
    g = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w)
    ref = R.layer_norm_bwd(R.d64(dy), R.d64(x), R.d64(f["mean"]), R.d64(f["rstd"]), R.d64(w), None)
    for k in ("x", "weight", "bias"):
        R.close("d" + k, g[k], *ref[k])
    if n == 0:
        assert (g["weight"] == 0).all() and (g["bias"] == 0).all()
    again = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w)
    assert all(torch.equal(g[k], again[k]) for k in g)  # sums in a fixed order


def test_layer_norm_gradient_against_differences(api):
    n, d = 6, 33
    x, dy = rand(1, n, d, torch.float32), rand(2, n, d, torch.float32)
    w, b = rand(3, 1, d, torch.float32)[0], rand(4, 1, d, torch.float32)[0]
    f = api.layer_norm(x, w, b)
    g = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w)
    X, W, B, DY = R.d64(x), R.d64(w), R.d64(b), R.d64(dy)
    loss = lambda X, W, B: (R.layer_norm(X, W, B, 1e-5)[0] * DY).sum().item()
    gen = torch.Generator().manual_seed(9)
    for _ in range(5):
        vx, vw, vb = (torch.randn(t.shape, generator=gen, dtype=R.F64) for t in (X, W, B))
        h = 1e-5
        diff = (loss(X + h * vx, W + h * vw, B + h * vb) - loss(X - h * vx, W - h * vw, B - h * vb)) / (2 * h)
        along = ((R.d64(g["x"]) * vx).sum() + (R.d64(g["weight"]) * vw).sum() + (R.d64(g["bias"]) * vb).sum()).item()
        terms = ((R.d64(g["x"]) * vx).abs().sum() + (R.d64(g["weight"]) * vw).abs().sum()).item()
        assert abs(diff - along) <= 1e-5 * terms, (diff, along)


def test_layer_norm_bad_rows_stay_in_their_rows(api):
    """An infinity or NaN spoils its own row; a constant row gives the bias."""
    n, d = 9, 100
    x = rand(1, n, d, torch.float32)
    clean = api.layer_norm(x)["y"].clone()
    x[2, 5], x[4, 0], x[6, 99] = float("inf"), float("nan"), -float("inf")
    x[7] = 3.0
    b = rand(3, 1, d, torch.float32)[0]
    y = api.layer_norm(x)["y"]
    assert y[[2, 4, 6]].isnan().all()
    keep = [0, 1, 3, 5, 8]
    assert torch.equal(y[keep], clean[keep])
    assert (y[7] == 0).all()
    assert torch.equal(api.layer_norm(x, None, b)["y"][7], b)


def test_layer_norm_in_place_and_partial_gradients(api):
    n, d = 50, 96
    x, dy = rand(1, n, d, torch.bfloat16), rand(2, n, d, torch.bfloat16)
    w = rand(3, 1, d, torch.bfloat16)[0]
    f = api.layer_norm(x, w)
    g = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w, add=dy)
    dy2 = dy.clone()
    r = api.layer_norm_bwd(dy2, x, f["mean"], f["rstd"], w, add=dy2, grads=dict(x=dy2))
    assert torch.equal(r["x"], g["x"]) and r["x"] is dy2
    only = dict(weight=torch.empty_like(w))
    api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w, grads=only)
    assert torch.equal(only["weight"], g["weight"])
    x2 = x.clone()
    assert torch.equal(api.layer_norm(x2, w, out=x2)["y"], f["y"])


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,d", [(0, 5), (1, 1), (3, 2), (5, 4), (17, 59), (9, 64), (4, 300), (2, 2051)])
def test_dropout_mask_and_values(api, dtype, n, d):
    seed, offset = 0xFEDCBA9876543210, (5 << 32) + 77
    for pad, skip in ((0, 0), (5, 1)):
        x, res = rand(1, n, d, dtype, pad, skip), rand(2, n, d, dtype, skip, pad)
        for p in (0.0, 0.1, 0.5, 1.0):
            say("dropout", dtype, n, d, pad, p)
            y = api.dropout(x, p, seed, offset)
            ref = R.dropout(R.d64(x), p, seed, offset)
            R.close("y", y, ref, ref.abs())
            assert torch.equal(d0(y), d0(api.dropout_bwd(x, p, seed, offset)))
            R.close("y + residual", api.dropout(x, p, seed, offset, residual=res), R.d64(res) + ref,
                    R.d64(res).abs() + ref.abs())
            z = res.clone()
            api.dropout(x, p, seed, offset, residual=z, out=z)
            assert torch.equal(z, api.dropout(x, p, seed, offset, residual=res))


def d0(t):
    return t.contiguous()


def test_dropout_removes_infinities_and_nan(api):
    x = torch.full((64, 40), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = api.dropout(x, 0.5, 11, 3)
    keep = R.keep_mask(64, 40, 0.5, 11, 3).cuda()
    assert (y[~keep] == 0).all()
    assert y[::2][keep[::2]].isinf().all() and y[1::2][keep[1::2]].isnan().all()
    assert (api.dropout(x, 1.0, 11, 3) == 0).all()


def test_dropout_rate_and_independence(api):
    """The kept share of 4M elements within 5 standard deviations; another seed
    or offset gives a mask that agrees with this one as chance has it."""
    n, d, p = 65536, 64, 0.3
    x = torch.ones(n, d, device="cuda")
    a = api.dropout(x, p, 1, 0) != 0
    tot = n * d
    assert abs(a.sum().item() - tot * (1 - p)) <= 5 * math.sqrt(tot * p * (1 - p))
    same = p * p + (1 - p) ** 2
    for seed, offset in ((2, 0), (1, 1), (1, 1 << 32), (1 + (1 << 32), 0)):
        b = api.dropout(x, p, seed, offset) != 0
        assert abs((a == b).sum().item() - tot * same) <= 5 * math.sqrt(tot * same * (1 - same)), (seed, offset)


def test_rows_past_32_bits_of_elements(api):
    """The last rows of a matrix of more than 2^32 elements."""
    n, d = (1 << 25) + 3, 130
    say("past 32 bits", n, d)
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    x[:4] = rand(1, 4, d, torch.bfloat16)
    x[4:-4] = 1.0
    x[-4:] = rand(2, 4, d, torch.bfloat16)
    y = api.layer_norm(x)["y"]
    ref = api.layer_norm(torch.cat((x[:4], x[-4:])))["y"]
    assert torch.equal(torch.cat((y[:4], y[-4:])), ref)
    del y
    z = api.dropout(x, 0.5, 3, 4)
    keep = torch.from_numpy(_mask_of_row(n - 1, d, 0.5, 3, 4)).cuda()
    assert torch.equal(z[-1], torch.where(keep, 2 * x[-1], torch.zeros_like(x[-1])))


def _mask_of_row(row, d, p, seed, offset):
    import numpy as np
    M, out = 0xFFFFFFFF, []
    for q in range((d + 3) // 4):
        c, k = [q, row, offset & M, offset >> 32], [seed & M, seed >> 32]
        for _ in range(7):
            a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [(b >> 32) ^ c[1] ^ k[0], b & M, (a >> 32) ^ c[3] ^ k[1], a & M]
            k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
        out += [w >= math.floor(p * 2 ** 32) for w in c]
    return np.array(out[:d])


def test_rows_on_a_side_stream(api):
    s = torch.cuda.Stream()
    x = rand(1, 3000, 64, torch.float32)
    ref = api.dropout(api.layer_norm(x)["y"], 0.2, 1, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        y = api.dropout(api.layer_norm(x)["y"], 0.2, 1, 2)
    s.synchronize()
    assert torch.equal(y, ref)


def test_refusals(api):
    x = rand(1, 8, 16, torch.float32)
    w = torch.ones(16, device="cuda")
    f = api.layer_norm(x, w)
    bad = [
        lambda: api.layer_norm(x.cpu()),
        lambda: api.layer_norm(x.double()),
        lambda: api.layer_norm(x[0]),
        lambda: api.layer_norm(x.t()),
        lambda: api.layer_norm(x[:, :0]),
        lambda: api.layer_norm(x[0].expand(8, 16)),
        lambda: api.layer_norm(x, w[:8]),
        lambda: api.layer_norm(x, w.half()),
        lambda: api.layer_norm(x, w, w.half()),
        lambda: api.layer_norm(x, out=torch.empty(8, 17, device="cuda")),
        lambda: api.layer_norm(x, mean=torch.empty(7, device="cuda")),
        lambda: api.layer_norm(x, eps=-1.0),
        lambda: api.layer_norm(x, eps=float("nan")),
        lambda: api.layer_norm_bwd(x.half(), x, f["mean"], f["rstd"], w),
        lambda: api.layer_norm_bwd(x[:4], x, f["mean"], f["rstd"], w),
        lambda: api.layer_norm_bwd(x, x, f["mean"].double(), f["rstd"], w),
        lambda: api.layer_norm_bwd(x, x, None, f["rstd"], w),
        lambda: api.layer_norm_bwd(x, x, f["mean"], f["rstd"], w, workspace=torch.empty(4, dtype=torch.uint8, device="cuda")),
        lambda: api.dropout(x, 1.5, 0),
        lambda: api.dropout(x, float("nan"), 0),
        lambda: api.dropout(x, 0.5, -1),
        lambda: api.dropout(x, 0.5, 0, 1 << 64),
        lambda: api.dropout(x, 0.5, 0, residual=x[:, :8]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, api.AbcdError)):
            call()
            print("not refused:", i)


def test_offsets_past_32_bits(api):
    """Rows so far apart that the last lie more than 2^31 elements (2^32 bytes) in."""
    n, d, ld = 2300, 67, 1 << 20
    for dtype in (torch.bfloat16, torch.float32):
        wide, into = (torch.empty((n, ld), dtype=dtype, device="cuda") for _ in range(2))
        x, y = wide[:, 5:5 + d], into[:, 3:3 + d]
        x.copy_(rand(1, n, d, dtype))
        near, dy = x.clone(), rand(2, n, d, dtype)
        f, g = api.layer_norm(x, out=y), api.layer_norm(near)
        assert torch.equal(y, g["y"]) and torch.equal(f["mean"], g["mean"])
        w = rand(3, 1, d, dtype)[0].contiguous()
        a = api.layer_norm_bwd(dy, x, g["mean"], g["rstd"], w, add=x)
        b = api.layer_norm_bwd(dy, near, g["mean"], g["rstd"], w, add=near)
        assert all(torch.equal(a[k], b[k]) for k in a if a[k] is not None)
        api.dropout(x, 0.3, 1, 2, residual=x, out=y)
        assert torch.equal(y, api.dropout(near, 0.3, 1, 2, residual=near))


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,d", [(1, 8200), (3, 20001), (40, 8200), (5, 4100), (50, 300), (9, 1500)])
def test_layer_norm_gradients_in_place(api, dtype, n, d):
    """dx written over dy, or over what is added to it, with every gradient wanted."""
    say("in place", dtype, n, d)
    x, dy, add = (rand(i, n, d, dtype) for i in (1, 2, 4))
    w = rand(3, 1, d, dtype)[0]
    f = api.layer_norm(x, w)
    for aa in (None, add):
        want = api.layer_norm_bwd(dy, x, f["mean"], f["rstd"], w, add=aa)
        for into in ("dy", "add")[:1 if aa is None else 2]:
            over = dict(dy=dy.clone(), add=None if aa is None else aa.clone())
            grads = dict(x=over[into], weight=torch.empty_like(w), bias=torch.empty_like(w))
            api.layer_norm_bwd(over["dy"], x, f["mean"], f["rstd"], w, add=over["add"], grads=grads)
            assert all(torch.equal(grads[k], want[k]) for k in want), into


def test_layer_norm_statistics_of_infinite_rows(api):
    """The mean of a row with an infinity is that infinity, with both NaN."""
    inf = float("inf")
    for dtype in DT:
        for d in (40, 4100, 20001):
            x = rand(1, 6, d, dtype)
            x[1, 3], x[2, d - 1], x[3, 0], x[3, 5], x[4, 7] = inf, -inf, inf, -inf, float("nan")
            f = api.layer_norm(x)
            assert f["mean"][1] == inf and f["mean"][2] == -inf and f["mean"][3:5].isnan().all()
            assert f["rstd"][1:5].isnan().all() and f["y"][1:5].isnan().all()
            assert f["mean"][[0, 5]].isfinite().all() and f["y"][[0, 5]].isfinite().all()


def test_layer_norm_of_tiny_rows(api):
    """With eps = 0 or a subnormal one the variance may be subnormal."""
    n, d, scale = 20, 96, 2.0 ** -66
    x = rand(1, n, d, torch.float32, scale=scale)
    for eps in (0.0, 2.0 ** -131):
        f = api.layer_norm(x, eps=eps)
        y, mean, rstd, mag = R.layer_norm(R.d64(x), None, None, eps)
        # every square and sum below 2^-126 is off by half of 2^-149 at most
        var = R.d64(x).var(1, unbiased=False)
        off = 4 * 2.0 ** -150 / (var + eps)
        assert ((R.d64(f["rstd"]) - rstd).abs() <= rstd * (16 * R.E32 + off)).all()
        assert ((R.d64(f["y"]) - y).abs() <= mag * (16 * R.E32 + off[:, None])).all()
