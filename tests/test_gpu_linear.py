"""The linear layer, forward and backward, against its float64 definition.
Tolerances: one rounding of the output, six standard deviations of what rounding
dz (and the slopes where they are kept) leaves, and fp32 roundings of the sums'
terms (16 of their magnitude)."""
import math

import pytest
import torch

import decoder_ref as D
import features_ref as R
from test_gpu_features import DT, IDS, rand, say

pytestmark = pytest.mark.gpu
ACTS = [None, "silu", "gelu", "relu", "sigmoid"]


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_27735_amd import api
    return api


def run(api, n, i, o, dtype, act, bias=True, res=True, pad=0, skip=0):
    say("linear", n, i, o, dtype, act, "bias" if bias else "", "pad", pad, skip)
    x, w = rand(1, n, i, dtype, pad, skip), rand(2, o, i, dtype, scale=i ** -0.5).contiguous()
    b = rand(3, 1, o, dtype, scale=0.3)[0] if bias else None
    r = rand(4, n, o, dtype, skip, pad) if res else None
    dy = rand(5, n, o, dtype, pad, 2 * skip)
    x64, w64, b64, dy64, u = D.d64(x), D.d64(w), D.d64(b), D.d64(dy), D.UNIT[dtype]
    # the slopes': half a step of their root's code is 1 / (30,800 root) of a slope, below 2^-11
    # of it above 2^-7 and, further down, below 2^-11 of it and 2^-19 together
    us = 0.0 if act is None else D.UNIT[torch.float32 if dtype == torch.float32 else torch.float16]
    f = api.linear(x, w, b, act, residual=r, save=True)
    y, my = R.linear(x64, w64, b64, act, D.d64(r))
    D.close("y", f["y"], y, my)
    assert (f["saved"] is not None) == (act is not None)
    assert torch.equal(api.linear(x, w, b, act, residual=r)["y"], f["y"])
    if res:  # onto the residual itself
        own = r.clone()
        assert api.linear(x, w, b, act, residual=own, out=own)["y"] is own and torch.equal(own, f["y"])
    names = {"x", "w"} | ({"b"} if bias else set())

    def check(got, ref, what):
        assert set(got) == names
        for k, v in got.items():
            D.close(what + " d" + k, v, ref[k][0], ref[k][1], extra=6 * ref[k][2])

    check(api.linear_bwd(dy, x, w, b, act), R.linear_bwd(dy64, x64, w64, b64, act, u, 0.0), "made again")
    kept = api.linear_bwd(dy, x, w, b, act, saved=f["saved"])
    check(kept, R.linear_bwd(dy64, x64, w64, b64, act, u, us), "kept")
    packed = api.pack8(x)
    x8 = D.d64(api.unpack8(packed))
    eight = api.linear_bwd(dy, packed, w, b, act)
    check(eight, R.linear_bwd(dy64, x8, w64, b64, act, u, 0.0), "8 bits")
    if act is not None:
        got = api.linear_bwd(dy, packed, w, b, act, saved=f["saved"])
        assert torch.equal(got["x"], kept["x"])  # x is in the weights' gradient only
        z = x64 @ w64.T + (0 if b is None else b64)
        dz = dy64 * R.act(z, act)[1]
        sdz = (u + us) * dz.abs() + us * 2.0 ** -8 * dy64.abs() + 16 * D.E32 * dy64.abs() * (1 + x64.abs() @ w64.abs().T)
        if act == "relu":
            sdz = sdz + torch.where(z.abs() <= 16 * D.E32 * (x64.abs() @ w64.abs().T + 1), dy64.abs(), torch.zeros_like(z))
        D.close("8 bits, kept dw", got["w"], dz.T @ x8, dz.abs().T @ x8.abs(), extra=6 * ((sdz ** 2).T @ x8 ** 2).sqrt())
    return x, w, b, dy, f, kept


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,i,o", [
    (1, 1, 1), (1, 8, 16), (2, 7, 3), (3, 64, 64), (17, 59, 48), (64, 96, 59), (65, 40, 65), (127, 130, 131), (128, 128, 128),
    (129, 257, 120), (300, 63, 257), (1100, 72, 48)])
def test_layer_sizes(api, dtype, n, i, o):
    run(api, n, i, o, dtype, "silu")
    run(api, n, i, o, dtype, None, bias=False, res=False, pad=3, skip=1)
    run(api, n, i, o, dtype, "gelu", res=False, pad=8)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("act", ACTS)
def test_activations(api, dtype, act):
    run(api, 70, 48, 40, dtype, act)
    run(api, 3000, 64, 64, dtype, act)
    run(api, 9, 300, 77, dtype, act, bias=False)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
def test_large_tiles_and_split_rows(api, dtype):
    """Enough tiles for the large ones in every product; long rows for the splits."""
    run(api, 6200, 2000, 2000, dtype, "silu")
    run(api, 9001, 24, 200, dtype, "gelu")


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,i,o", [
    (1024, 64, 64), (1025, 1, 1), (2049, 7, 5), (2049, 33, 48), (3000, 59, 61), (1500, 16, 128), (1500, 128, 16), (20011, 64, 64),
    (70001, 24, 50), (4099, 128, 64), (4100, 64, 128), (5001, 121, 63), (3001, 128, 128), (2500, 96, 59),
    (1003, 256, 128), (1500, 200, 72), (900, 131, 63), (1001, 250, 3), (777, 64, 256), (1200, 127, 201), (65, 17, 129)])
def test_narrow_rows(api, dtype, n, i, o):
    run(api, n, i, o, dtype, "silu")
    run(api, n, i, o, dtype, None, bias=False, res=False, pad=5, skip=1)


@pytest.mark.parametrize("n", [2, 8, 16, 31, 33, 64])
@pytest.mark.parametrize("i,o", [(512, 1376), (1001, 333)])
def test_few_rows(api, n, i, o):
    run(api, n, i, o, torch.float16, "silu")
    run(api, n, i, o, torch.bfloat16, "sigmoid", bias=False, pad=8)
    run(api, n, i, o, torch.float32, "gelu", res=False)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,i,o", [(1, 40, 2101), (17, 72, 2049), (3, 33, 4999), (16, 8, 6145)])
def test_few_rows_of_many_columns(api, dtype, n, i, o):
    run(api, n, i, o, dtype, "gelu")
    run(api, n, i, o, dtype, None, pad=3, skip=1)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,i,o", [(137, 1024, 520), (70, 600, 2100), (65, 4000, 9), (200, 33, 3001), (300, 2515, 260)])
def test_few_tiles_and_long_sums(api, dtype, n, i, o):
    run(api, n, i, o, dtype, "silu")
    run(api, n, i, o, dtype, None, pad=3, skip=1)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,i,o", [(5, 40, 24), (2000, 64, 40), (700, 300, 200)])
def test_gradients_one_by_one(api, dtype, n, i, o):
    x, w, b, dy, f, _ = run(api, n, i, o, dtype, "silu")
    for saved in (f["saved"], None):
        want = api.linear_bwd(dy, x, w, b, "silu", saved=saved)
        for k in want:
            out = torch.full_like(want[k], math.nan)
            got = api.linear_bwd(dy, x, w, b, "silu", saved=saved, grads={k: out})
            assert set(got) == {k} and got[k] is out and torch.equal(out, want[k]), k
        for _ in range(2):
            again = api.linear_bwd(dy, x, w, b, "silu", saved=saved)
            assert all(torch.equal(again[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
def test_layer_of_no_rows(api, dtype):
    x, w, b = torch.zeros(0, 40, dtype=dtype, device="cuda"), torch.ones(24, 40, dtype=dtype, device="cuda"), torch.ones(24, dtype=dtype, device="cuda")
    f = api.linear(x, w, b, "silu", save=True)
    assert f["y"].shape == (0, 24)
    for saved in (f["saved"], None):
        for rows in (x, api.pack8(x)):
            g = api.linear_bwd(f["y"], rows, w, b, "silu", saved=saved)
            assert g["x"].shape == (0, 40) and (g["w"] == 0).all() and (g["b"] == 0).all()


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
@pytest.mark.parametrize("n,i,o", [(40, 64, 64), (3000, 64, 64), (300, 200, 300)])
def test_not_finite_rows_stay_by_themselves(api, dtype, n, i, o):
    """Rows that hold an infinity or a NaN reach no other row of y, dx and the slopes, and rows
    behind the last one are left as they were."""
    x, w, b = rand(1, n, i, dtype), rand(2, o, i, dtype, scale=i ** -0.5).contiguous(), rand(3, 1, o, dtype)[0]
    dy = rand(5, n, o, dtype)
    clean, gclean = api.linear(x, w, b, "silu")["y"], api.linear_bwd(dy, x, w, b, "silu")["x"]
    x[7, 3], x[20] = math.inf, math.nan
    room = torch.full((n + 3, o), 5.0, dtype=dtype, device="cuda")
    y = api.linear(x, w, b, "silu", out=room[:n])["y"]
    rooms = torch.full((n + 3, i), 5.0, dtype=dtype, device="cuda")
    api.linear_bwd(dy, x, w, b, "silu", grads=dict(x=rooms[:n]))
    fine = [r for r in range(n) if r not in (7, 20)]
    assert torch.equal(y[fine], clean[fine]) and torch.equal(rooms[:n][fine], gclean[fine])
    assert y[20].isnan().all() and (room[n:] == 5).all() and (rooms[n:] == 5).all()


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
def test_far_rows(api, dtype):
    """Rows more than 2^31 elements apart."""
    ld = (1 << 30) + 8
    far = torch.empty(2 * ld + 64, dtype=dtype, device="cuda").as_strided((3, 64), (ld, 1))
    x, w, dy = rand(1, 3, 64, dtype), rand(2, 64, 64, dtype).contiguous(), rand(3, 3, 64, dtype)
    want, g = api.linear(x, w, act="silu")["y"], api.linear_bwd(dy, x, w, act="silu")
    far.copy_(x)
    assert torch.equal(api.linear(far, w, act="silu")["y"], want)
    got = api.linear_bwd(dy, far, w, act="silu")
    assert all(torch.equal(got[k], g[k]) for k in g)
    api.linear(x, w, act="silu", out=far)
    assert torch.equal(far, want)
    far.copy_(dy)
    got = api.linear_bwd(far, x, w, act="silu")
    assert all(torch.equal(got[k], g[k]) for k in g)
    api.linear_bwd(dy, x, w, act="silu", grads=dict(x=far))
    assert torch.equal(far, g["x"])


def test_linear_refuses(api):
    x, w, b = torch.zeros(4, 16, device="cuda"), torch.zeros(8, 16, device="cuda"), torch.zeros(8, device="cuda")
    dy, p = torch.zeros(4, 8, device="cuda"), api.pack8(torch.zeros(4, 16, device="cuda"))
    s = api.linear(x, w, b, "silu", save=True)["saved"]
    bad = [lambda: api.linear(x, w, b, "tanh"), lambda: api.linear(x.double(), w), lambda: api.linear(x, w.half()),
           lambda: api.linear(x, w[:, :15]), lambda: api.linear(x, w.t()), lambda: api.linear(x, w[:0]), lambda: api.linear(x, w, b[:7]),
           lambda: api.linear(x, w, b.half()), lambda: api.linear(x, w, residual=x), lambda: api.linear(x, w, out=x),
           lambda: api.linear(x.cpu(), w), lambda: api.linear(x[0], w), lambda: api.linear(x.t(), w), lambda: api.linear(p, w),
           lambda: api.linear_bwd(x, x, w), lambda: api.linear_bwd(dy.half(), x, w), lambda: api.linear_bwd(dy[:3], x, w),
           lambda: api.linear_bwd(dy, p._replace(dtype=torch.float16), w), lambda: api.linear_bwd(dy, p._replace(width=15), w),
           lambda: api.linear_bwd(dy, x, w, act="silu", saved=s[:3]), lambda: api.linear_bwd(dy, x, w, act="silu", saved=s.half()),
           lambda: api.linear_bwd(dy, x, w, grads=dict(w=w.t())), lambda: api.linear_bwd(dy, x, w, grads=dict(x=dy)),
           lambda: api.linear_bwd(dy, x, w, b, grads=dict(b=b[:3]))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    many = torch.zeros(400, 16, device="cuda")  # (of few rows none is needed)
    with pytest.raises(api.AbcdError):
        api.linear(many, w, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    with pytest.raises(api.AbcdError):
        api.linear_bwd(dy, x, w, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("act", [None, "relu"])
@pytest.mark.parametrize("n,i,o", [(40, 64, 64), (300, 70, 24), (5, 33, 9), (70, 128, 60), (90, 40, 300)])
def test_checkpoint_of_the_largest_numbers(api, dtype, act, n, i, o):
    """A block whose exponent is the type's largest stands for the same numbers in the layer's
    gradients as unpacked. (One number of that size a row, so that no sum leaves the type, and
    the sign of z, which ReLU's slope goes by, is that of its product.)"""
    x = rand(1, n, i, dtype)
    x[:, 5] = torch.finfo(dtype).max * (1.0 - 2.0 * (torch.arange(n) % 2)).cuda()
    w = rand(2, o, i, dtype, scale=i ** -0.5).contiguous()
    w[:, 5] = torch.where(w[:, 5] < 0, -0.25, 0.25)
    dy = (2.0 ** -10 * (1 + (torch.arange(n * o) * 7 % 3).view(n, o))).to(dtype).cuda()
    packed = api.pack8(x)
    rows = api.unpack8(packed)
    assert torch.isfinite(rows).all() and (rows[:, 5].abs() > 0.98 * torch.finfo(dtype).max).all()
    got, want = api.linear_bwd(dy, packed, w, act=act), api.linear_bwd(dy, rows, w, act=act)
    x8, w64, dy64 = D.d64(rows), D.d64(w), D.d64(dy)
    assert torch.equal(got["x"], want["x"])
    dz = dy64 if act is None else dy64 * ((x8 @ w64.T) > 0)
    D.close("dw", got["w"], dz.T @ x8, dz.abs().T @ x8.abs())
    D.close("dx", got["x"], dz @ w64, dz.abs() @ w64.abs())


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
@pytest.mark.parametrize("act", ["silu", "sigmoid", "relu"])
@pytest.mark.parametrize("n,i,o", [(1, 512, 1376), (2, 300, 1001), (16, 512, 1376), (17, 200, 333), (31, 512, 1376), (33, 300, 1001),
                                   (48, 512, 1376), (64, 300, 2050)])
def test_bias_gradient_of_few_rows(api, dtype, act, n, i, o):
    """Where the slopes of a few rows are made again the bias's gradient is the sum of dz before it
    is rounded, as it is with slopes that were kept: nothing but its own rounding, and the fp32 sums'."""
    x, w, b, dy = rand(1, n, i, dtype), rand(2, o, i, dtype, scale=i ** -0.5).contiguous(), rand(3, 1, o, dtype)[0], rand(4, n, o, dtype)
    for rows in (x, api.pack8(x)):
        x64 = D.d64(rows if rows is x else api.unpack8(rows))
        ref, mag, sd = R.linear_bwd(D.d64(dy), x64, D.d64(w), D.d64(b), act, 0.0, 0.0)["b"]
        whole = api.linear_bwd(dy, rows, w, b, act)
        D.close("db", whole["b"], ref, mag, extra=6 * sd)
        alone = api.linear_bwd(dy, rows, w, b, act, grads=dict(b=torch.full_like(b, math.nan)))["b"]
        assert torch.equal(alone, whole["b"])


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
@pytest.mark.parametrize("n,i", [(16, 64), (200, 64), (200, 300)])
def test_kept_slopes_of_a_tail(api, dtype, n, i):
    """The code of a kept slope s holds its root in steps of 1 / 30,800, so that s is off by no
    more than sqrt(s) / 30,800 and a quarter of a step squared. With w the identity and dy ones dx
    is s, rounded once as dz and unchanged by the product with ones and zeros."""
    x = torch.linspace(-12.0, -4.0, n * i).view(n, i).to(dtype).cuda()
    w, dy = torch.eye(i, dtype=dtype, device="cuda"), torch.ones(n, i, dtype=dtype, device="cuda")
    saved = api.linear(x, w, act="sigmoid", save=True)["saved"]
    s = R.act(D.d64(x), "sigmoid")[1]
    got = D.d64(api.linear_bwd(dy, x, w, act="sigmoid", saved=saved)["x"])
    # and in fp32 by the exponent rounded at a z of 12, and 12 more for exponentials, reciprocals and product
    code = s.sqrt() / 30800 + 0.25 / 30800 ** 2 + 24 * D.E32 * s
    u = D.UNIT[dtype]
    assert ((got - s).abs() <= u * s + D.TINY[dtype] + (1 + u) * code).all()


@pytest.mark.parametrize("n,i,o", [(40, 64, 64), (3000, 64, 64), (300, 200, 300)])
def test_not_finite_rows_of_float32(api, n, i, o):
    test_not_finite_rows_stay_by_themselves(api, torch.float32, n, i, o)


def test_far_rows_of_float32(api):
    test_far_rows(api, torch.float32)


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
def test_weight_gradient_of_large_tiles(api, dtype):
    """260 tiles of 256 x 256: a round of the GPU, and four whose rows are split into parts
    that the kernel for many of them adds up; the last tile of each side is not whole."""
    n, i, o = 8200, 256 * 13 - 8, 256 * 20 - 24
    say("dw", n, i, o, dtype)
    x, dy = rand(1, n, i, dtype), rand(2, n, o, dtype)
    w = torch.zeros(o, i, dtype=dtype, device="cuda")
    dw = torch.full_like(w, math.nan)
    api.linear_bwd(dy, x, w, grads=dict(w=dw))
    # a row of every tile, and the last ones; fp32 sums of 8,200 terms: 128 indexes a step, one
    # product's sum after the other (257 of 32 terms), or parts of fewer and their sum
    rows = torch.tensor([256 * k + 37 * k % 256 for k in range(19)] + [256 * 19 + 5, o - 1])
    dy64, x64 = D.d64(dy[:, rows.cuda()]), D.d64(x)
    D.close("dw", dw[rows.cuda()], dy64.T @ x64, dy64.abs().T @ x64.abs(), k=300.0)


@pytest.mark.parametrize("dtype", DT[1:], ids=IDS[1:])
def test_layer_of_small_tiles_by_rounds(api, dtype):
    """288 large tiles, whose second round would be nearly empty: the small ones take it."""
    n, i, o = 6000, 3000, 3000
    say("linear", n, i, o, dtype)
    x, w, b, r = rand(1, n, i, dtype), rand(2, o, i, dtype, scale=i ** -0.5).contiguous(), rand(3, 1, o, dtype)[0], rand(4, n, o, dtype)
    y = api.linear(x, w, b, "silu", residual=r)["y"]
    rows = torch.tensor([0, 127, 128, 255, 2999, 5887, 5888, 5999])
    at = rows.cuda()
    ref, mag = R.linear(D.d64(x[at]), D.d64(w), D.d64(b), "silu", D.d64(r[at]))
    D.close("y", y[at], ref, mag, k=110.0)  # 94 products' sums one after the other, the bias, act and residual
