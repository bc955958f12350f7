"""The joint between two blocks against its float64 definition, forward and
backward, at every row shape of its kernels, with every pair of norms, kind of gate
and set of parameters. Tolerances: one rounding to the output's type and 64 fp32
roundings of the magnitude of the terms behind it (a lane adds up to 16 numbers of a row,
the lanes and waves up to 10 sums in turn; a column of these tests at most 32 rows one
after the other, and up to 16 waves' and 16 parts' sums)."""
import math

import pytest
import torch

import decoder_ref as D
import features_ref as R
from test_gpu_features import DT, IDS, rand, say

pytestmark = pytest.mark.gpu
K = 64.0


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_27735_amd import api
    return api


def make(n, d, dtype, post, pre, gate, scale=True, wtype=None, pad=0, skip=0, bare=False, seed=0):
    """Inputs of a joint: f, x, its parameters and its gate."""
    wtype = wtype or dtype
    f = rand(seed + 1, n, d, dtype, pad, skip, scale=1.5, shift=0.4)
    x = rand(seed + 2, n, d, dtype, 2 * pad, skip)
    p = {}
    vec = lambda s, scale, shift: rand(seed + s, 1, d, wtype, scale=scale, shift=shift)[0]
    if not bare:
        for k, kind, s in (("post", post, 3), ("pre", pre, 5)):
            if kind:
                p[k + "_weight"] = vec(s, 0.3, 1.0)
            if kind == "layer":
                p[k + "_bias"] = vec(s + 1, 0.3, 0.0)
    if scale:
        p["scale"] = vec(7, 0.2, 0.5)
    g = None if gate == "none" else rand(seed + 8, n, 1 if gate == "row" else d, dtype, pad + (gate == "row"), skip, scale=0.4, shift=0.5)
    return f, x, p, g


def check(api, n, d, dtype, post, pre, gate, eps=1e-5, with_dy=True, **kw):
    f, x, p, g = make(n, d, dtype, post, pre, gate, **kw)
    call = dict(post=post, pre=pre, params=p, gate=g)
    r = api.residual_norm(f, x, eps=eps, **call)
    p64, g64 = {k: D.d64(v) for k, v in p.items()}, D.d64(g)
    ref = R.residual_norm(D.d64(f), D.d64(x), post, pre, p64, g64, eps)
    for k in ("y", "z", "post_mean", "post_rstd", "pre_mean", "pre_rstd"):
        assert (r[k] is not None) == (k in ref), k
        if k in ref:
            D.close(k, r[k], ref[k][0], ref[k][1], k=K)
    pad, skip = kw.get("pad", 0), kw.get("skip", 0)
    dz = rand(11, n, d, dtype, pad, skip) if pre else None
    dy = rand(12, n, d, dtype, 2 * pad, skip) if with_dy else None
    got = api.residual_norm_bwd(dz, dy, f, r, **call)
    stats = {k: D.d64(r[k]) for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd") if r[k] is not None}
    want = R.residual_norm_bwd(D.d64(dz), D.d64(dy), D.d64(f), D.d64(r["y"]), stats, post, pre, p64, g64)
    assert set(got) == {"x", "f"} | set(p) | ({"gate"} if g is not None else set())
    for k, v in got.items():
        D.close(k, v, want[k][0], want[k][1], k=K)
    # the same again into tensors that are there, and each by itself
    again = api.residual_norm_bwd(dz, dy, f, r, grads={k: torch.full_like(v, math.nan) for k, v in got.items()}, **call)
    for k, v in got.items():
        assert torch.equal(again[k], v), k
        alone = api.residual_norm_bwd(dz, dy, f, r, grads={k: torch.full_like(v, math.nan)}, **call)
        assert set(alone) == {k} and torch.equal(alone[k], v), k
    return f, x, p, g, r, got


# every row shape (8 lanes to 1,024, rows read again), odd widths, one element
WIDTHS = [1, 2, 7, 16, 59, 64, 100, 129, 256, 500, 1001, 1024, 2048, 2053, 4096, 5000, 8192, 8200, 20001]


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("d", WIDTHS)
def test_joint_widths(api, dtype, d):
    n = 37 if d < 2000 else 5
    say("joint", dtype, n, d, "layer layer row")
    check(api, n, d, dtype, "layer", "layer", "row")
    say("joint", dtype, n, d, "rms rms full, strided, fp32 parameters")
    check(api, n, d, dtype, "rms", "rms", "full", wtype=torch.float32, pad=3, skip=1)


KINDS = [(a, b) for a in (None, "layer", "rms") for b in (None, "layer", "rms")]


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("gate", ["none", "row", "full"])
def test_joint_kinds(api, dtype, post, pre, gate):
    for n, d, scale, bare, with_dy in ((70, 96, True, False, True), (3, 700, False, False, pre is None), (9, 33, False, True, True)):
        say("joint", dtype, n, d, post, pre, gate, scale, bare, with_dy)
        check(api, n, d, dtype, post, pre, gate, scale=scale, bare=bare, with_dy=with_dy)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,d", [(1, 2048), (2, 64), (64, 64), (65, 64), (1000, 40), (8200, 17), (600, 1024), (300, 4096)])
def test_joint_row_counts(api, dtype, n, d):
    say("joint", dtype, n, d)
    check(api, n, d, dtype, "rms", "layer", "row")


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("d", [64, 1001, 20001])
def test_joint_odd_rows(api, dtype, d):
    """Constant rows, rows of zeros (1 / sd is that of eps), and rows that hold an infinity
    or a NaN, which reach no other row."""
    f, x, p, g = make(6, d, dtype, "layer", "rms", "row")
    clean = api.residual_norm(f, x, post="layer", pre="rms", params=p, gate=g)
    f[1], x[2], f[2] = 3.0, 0.0, 0.0
    f[3, d // 2], f[4, d - 1] = math.inf, math.nan
    g[5] = 0.0
    r = api.residual_norm(f, x, post="layer", pre="rms", params=p, gate=g)
    assert torch.equal(r["y"][0], clean["y"][0]) and torch.equal(r["z"][0], clean["z"][0])
    p64 = {k: D.d64(v) for k, v in p.items()}
    ref = R.residual_norm(D.d64(f), D.d64(x), "layer", "rms", p64, D.d64(g), 1e-5)
    for k in ("y", "z"):
        for i in (1, 2, 5):
            D.close(k, r[k][i], ref[k][0][i], ref[k][1][i], k=K)
        assert r[k][3:5].isnan().all()
    assert torch.equal(r["y"][5], x[5])  # a closed gate adds nothing
    dz, dy = rand(11, 6, d, dtype), rand(12, 6, d, dtype)
    got = api.residual_norm_bwd(dz, dy, f, r, post="layer", pre="rms", params=p, gate=g)
    assert (got["f"][5] == 0).all() and got["f"][3].isnan().all() and torch.isfinite(got["x"][[0, 1, 2, 5]]).all()


def test_joint_of_no_rows(api):
    f = torch.zeros(0, 64, device="cuda")
    p = {k: torch.ones(64, device="cuda") for k in ("post_weight", "pre_weight", "scale")}
    r = api.residual_norm(f, f, post="rms", pre="rms", params=p)
    assert r["y"].shape == (0, 64)
    g = api.residual_norm_bwd(f, f, f, r, post="rms", pre="rms", params=p)
    assert g["x"].shape == (0, 64) and all((g[k] == 0).all() for k in p)


def test_joint_far_rows(api):
    """Rows more than 2^31 elements apart."""
    ld = (1 << 30) + 8
    buf = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((3, 64), (ld, 1))
    f, x, p, g = make(3, 64, torch.bfloat16, "layer", "layer", "row")
    call = dict(post="layer", pre="layer", params=p, gate=g)
    r = api.residual_norm(f, x, **call)
    far.copy_(f)
    s = api.residual_norm(far, x, **call)
    assert all(torch.equal(s[k], r[k]) for k in r)
    dz, dy = rand(11, 3, 64, torch.bfloat16), rand(12, 3, 64, torch.bfloat16)
    want = api.residual_norm_bwd(dz, dy, f, r, **call)
    got = api.residual_norm_bwd(dz, dy, far, r, **call)
    assert all(torch.equal(got[k], want[k]) for k in want)
    api.residual_norm(f, x, out=far, **call)
    assert torch.equal(far, r["y"])
    api.residual_norm_bwd(dz, dy, f, r, grads=dict(x=far), **call)
    assert torch.equal(far, want["x"])


def test_joint_refuses(api):
    f, x, p, g = make(4, 16, torch.float32, "rms", "rms", "row")
    call = dict(post="rms", pre="rms", params=p, gate=g)
    r = api.residual_norm(f, x, **call)
    bwd = lambda **kw: api.residual_norm_bwd(**{**dict(dz=f, dy=f, f=f, kept=r), **call, **kw})
    bad = [lambda: api.residual_norm(f, x[:3]), lambda: api.residual_norm(f, x.half()), lambda: api.residual_norm(f, x, post="batch"),
           lambda: api.residual_norm(f, x, params=dict(weight=p["scale"])), lambda: api.residual_norm(f, x, params=dict(post_weight=p["scale"])),
           lambda: api.residual_norm(f, x, post="rms", params=dict(post_bias=p["scale"])),
           lambda: api.residual_norm(f, x, params=dict(scale=p["scale"][:3])), lambda: api.residual_norm(f, x, params=dict(scale=p["scale"].half())),
           lambda: api.residual_norm(f, x, gate=g[:, 0]), lambda: api.residual_norm(f, x, gate=f[:, :3]), lambda: api.residual_norm(f, x, gate=g.half()),
           lambda: api.residual_norm(f, x, z=f), lambda: api.residual_norm(f, x, out=f[:2]), lambda: api.residual_norm(f.cpu(), x),
           lambda: bwd(dz=None), lambda: bwd(pre=None, dz=None, dy=None, params=None), lambda: bwd(dy=f[:2]), lambda: bwd(kept=dict(r, pre_rstd=None)),
           lambda: bwd(kept=dict(r, post_rstd=r["post_rstd"][:2])), lambda: bwd(grads=dict(gate=f)), lambda: bwd(grads=dict(scale=f[0, :3])),
           lambda: bwd(gate=None, grads=dict(gate=g))]
    for call_ in bad:
        with pytest.raises(ValueError):
            call_()
    with pytest.raises(api.AbcdError):
        api.residual_norm(f, x, post="rms", eps=-1.0)
    with pytest.raises(api.AbcdError):
        bwd(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("n,d", [(5, 64), (3000, 64), (40, 1001), (5, 20001)])
def test_scale_gradient_of_infinite_rows(api, dtype, post, n, d):
    """An infinity in dy makes scale's gradient of its column that infinity, not a NaN, where
    the norm has no bias to multiply it with."""
    f, x, p, _ = make(n, d, dtype, post, None, "none")
    p.pop("post_bias", None)
    call = dict(post=post, params=p)
    r = api.residual_norm(f, x, **call)
    dy = rand(12, n, d, dtype)
    dy[3, 7], dy[n - 1, d - 2] = math.inf, -math.inf
    got = api.residual_norm_bwd(None, dy, f, r, grads=dict(scale=torch.empty_like(p["scale"])), **call)["scale"]
    stats = {k: D.d64(r[k]) for k in ("post_mean", "post_rstd") if r[k] is not None}
    want, mag = R.residual_norm_bwd(None, D.d64(dy), D.d64(f), None, stats, post, None, {k: D.d64(v) for k, v in p.items()}, None)["scale"]
    assert want.isinf().sum() == 2 and not want.isnan().any()
    D.close("scale", got, want, mag, k=K)


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("n,d", [(17000, 40), (2100, 700), (1100, 2048), (600, 4096), (300, 8200)])
def test_joint_rows_in_turns(api, dtype, n, d):
    """More rows than all workgroups take at once, at every way of holding a row."""
    say("joint", dtype, n, d)
    check(api, n, d, dtype, "layer", "layer", "full")


@pytest.mark.parametrize("dtype", DT, ids=IDS)
@pytest.mark.parametrize("gate", ["none", "row", "full"])
@pytest.mark.parametrize("n,d", [(6, 64), (9, 1001), (5, 20001)])
def test_gradients_of_infinite_rows_without_norms(api, dtype, gate, n, d):
    """Without a norm f has no part in its own gradient nor in x's: an infinity or a NaN in it
    leaves both as they are."""
    f, x, p, g = make(n, d, dtype, None, None, gate)
    f[1, 3], f[2], f[3, d - 1] = math.inf, math.nan, -math.inf
    call = dict(params=p, gate=g)
    r = api.residual_norm(f, x, **call)
    dy = rand(12, n, d, dtype)
    got = api.residual_norm_bwd(None, dy, f, r, **call)
    want = R.residual_norm_bwd(None, D.d64(dy), D.d64(f), None, {}, None, None, {k: D.d64(v) for k, v in p.items()}, D.d64(g))
    assert torch.isfinite(want["f"][0]).all()
    for k in ("x", "f"):
        D.close(k, got[k], want[k][0], want[k][1], k=K)
