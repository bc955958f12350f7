"""The entry points of the operators around a decoder's blocks refuse bad
arguments on the host, before any HIP call, and the float64 definitions of
their tests agree with differences."""
import ctypes as C
import os

import pytest
import torch

import decoder_ref as D
import features_ref as R

FAKE = 0x1000  # never dereferenced: every call below fails validation first
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2608_27735_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_27735_amd import build
        build.build()
    return _lib.load()


def refuse(base, call, cases):
    for i, v in cases:
        a = list(base)
        a[i] = v
        assert call(*a) == 1, (i, v)


def test_embed_refuses(lib):
    base = [F16, 4, 5, 8, F16, FAKE, 8, 32, FAKE, 1.0, FAKE, 8, None]
    refuse(base, lib.abcd_embed,
           [(0, 3), (1, -1), (1, (1 << 30) + 1), (2, 0), (2, (1 << 30) + 1), (3, 0), (3, 65537), (4, BF16),
            (5, None), (5, FAKE + 1), (6, 7), (7, 16), (8, None), (8, FAKE + 2), (9, float("inf")), (9, float("nan")), (10, None), (10, FAKE + 1), (11, 7)])
    base[7] = 64
    refuse(base, lib.abcd_embed, [(8, FAKE + 4)])


def test_embed_sort_refuses(lib):
    need = C.c_size_t(0)
    assert lib.abcd_embed_sort_workspace_size(4, 5, C.byref(need)) == 0 and need.value >= 4 * 4 * 2
    refuse([4, 5, C.byref(need)], lib.abcd_embed_sort_workspace_size, [(0, -1), (1, 0), (1, (1 << 30) + 1), (2, None)])
    base = [4, 5, 32, FAKE, FAKE, FAKE, FAKE, FAKE, need.value, None]
    refuse(base, lib.abcd_embed_sort,
           [(0, -1), (1, 0), (2, 8), (3, None), (3, FAKE + 2), (4, None), (4, FAKE + 2), (5, None), (5, FAKE + 2),
            (6, None), (6, FAKE + 4), (7, None), (7, FAKE + 16), (8, need.value - 1)])


def test_embed_bwd_refuses(lib):
    need = C.c_size_t(0)
    assert lib.abcd_embed_bwd_workspace_size(4, 8, C.byref(need)) == 0 and need.value >= 2 * 8 * 4
    refuse([4, 8, C.byref(need)], lib.abcd_embed_bwd_workspace_size, [(0, -1), (1, 0), (1, 65537), (2, None)])
    base = [BF16, 4, 5, 8, FAKE, 8, FAKE, FAKE, FAKE, 1.0, F32, FAKE, 8, FAKE, need.value, None]
    refuse(base, lib.abcd_embed_bwd,
           [(0, 7), (1, -1), (2, 0), (3, 0), (4, None), (4, FAKE + 1), (5, 7), (6, None), (6, FAKE + 1), (7, None),
            (8, None), (8, FAKE + 4), (9, float("inf")), (9, float("nan")), (10, F16), (11, None), (11, FAKE + 2), (12, 7), (13, None), (13, FAKE + 8),
            (14, need.value - 1)])


def test_embed_bwd_few_refuses(lib):
    base = [BF16, 4, 5, 8, FAKE, 8, 32, FAKE, 1.0, F32, FAKE, 8, None]
    refuse(base, lib.abcd_embed_bwd_few,
           [(0, 7), (1, -1), (1, 65), (2, 0), (3, 0), (4, None), (4, FAKE + 1), (5, 7), (6, 8), (7, None), (7, FAKE + 2),
            (8, float("inf")), (9, F16), (10, None), (10, FAKE + 2), (11, 7)])


def test_pack8_refuses(lib):
    base = [F16, 4, 8, FAKE, 8, FAKE, FAKE, None]
    refuse(base, lib.abcd_pack8, [(0, 3), (1, -1), (2, 0), (2, 65537), (3, None), (3, FAKE + 1), (4, 7), (5, None),
                                  (5, FAKE + 8), (6, None)])
    base = [F32, 4, 8, FAKE, FAKE, FAKE, 8, None]
    refuse(base, lib.abcd_unpack8, [(0, 3), (1, -1), (2, 0), (3, None), (3, FAKE + 8), (4, None), (5, None),
                                    (5, FAKE + 2), (6, 7)])


def test_python_refuses_what_is_not_on_the_gpu():
    from paper_2608_27735_amd import api
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: api.embed(x, i), lambda: api.embed_sort(i, 4), lambda: api.embed_bwd(x, i, 4),
                 lambda: api.embed_sort(i, 0), lambda: api.pack8(x),
                 lambda: api.unpack8(api.Packed8(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8),
                                                 8, torch.float32))):
        with pytest.raises(ValueError):
            call()


def test_reference_embed_gradient_is_its_forwards():
    g = torch.Generator().manual_seed(0)
    t = torch.randn(5, 3, generator=g, dtype=D.F64).requires_grad_()
    dy = torch.randn(9, 3, generator=g, dtype=D.F64)
    index = torch.tensor([0, 4, 4, -1, 2, 5, 0, 4, 2])
    inside = (index >= 0) & (index < 5)
    want, = torch.autograd.grad((t[index[inside]] * 1.5 * dy[inside]).sum(), t)
    assert torch.allclose(R.embed_bwd(dy, index, 5, 1.5)[0], want, rtol=1e-12)
    assert torch.allclose(R.embed(t.detach(), index, 1.5)[inside], t.detach()[index[inside]] * 1.5, rtol=1e-12)


def test_reference_checkpoint_keeps_within_its_step():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(7, 70, generator=g, dtype=D.F64) * torch.exp(3 * torch.randn(7, 70, generator=g, dtype=D.F64))
    y, e = R.pack8(x)
    top = torch.stack([x[:, b:b + 32].abs().amax(1) for b in (0, 32, 64)], 1)
    err = torch.stack([(y - x)[:, b:b + 32].abs().amax(1) for b in (0, 32, 64)], 1)
    assert (err <= top / 64).all() and (err <= 2.0 ** (e.to(D.F64) - 127 - 6)).all()
    assert torch.equal(R.pack8(y)[0], y)  # what was kept once is kept


def joint(**kw):
    from paper_2608_27735_amd import _lib
    j = dict(dtype=F16, wdtype=F16, post=1, pre=2, gate=1, eps=1e-5, d=8, post_weight=FAKE, post_bias=FAKE,
             pre_weight=FAKE, pre_bias=None, scale=FAKE)
    j.update(kw)
    return _lib.abcd_joint(*j.values())


BAD_JOINTS = [dict(dtype=3), dict(wdtype=BF16), dict(post=3), dict(post=-1), dict(pre=3), dict(gate=3), dict(eps=-1.0),
              dict(eps=float("nan")), dict(eps=float("inf")), dict(d=0), dict(d=65537), dict(post=0), dict(post=2),
              dict(pre=0), dict(pre_bias=FAKE), dict(scale=FAKE + 1), dict(post_weight=FAKE + 1)]


def test_residual_norm_refuses(lib):
    j = joint()
    base = [C.byref(j), 4, FAKE, 8, FAKE, 8, FAKE, 1, FAKE, 8, FAKE, 8, FAKE, FAKE, FAKE, FAKE, None]
    refuse(base, lib.abcd_residual_norm,
           [(0, None), (1, -1), (1, (1 << 30) + 1), (2, None), (2, FAKE + 1), (3, 7), (4, None), (5, 7), (6, None),
            (6, FAKE + 1), (7, 0), (8, None), (9, 7), (10, None), (11, 7), (12, FAKE + 2), (15, FAKE + 1)])
    refuse(base, lib.abcd_residual_norm, [(0, C.byref(joint(**kw))) for kw in BAD_JOINTS])
    # an element's gate has rows as wide as f's; no gate and no norm after it take no array
    refuse(base, lib.abcd_residual_norm, [(0, C.byref(joint(gate=2))), (0, C.byref(joint(gate=0))),
                                          (0, C.byref(joint(pre=0, pre_weight=None)))])


def test_residual_norm_bwd_refuses(lib):
    j, need = joint(), C.c_size_t(0)
    assert lib.abcd_residual_norm_bwd_workspace_size(C.byref(j), 4, C.byref(need)) == 0 and need.value >= 4 * 8 * 4
    refuse([C.byref(j), 4, C.byref(need)], lib.abcd_residual_norm_bwd_workspace_size,
           [(0, None), (1, -1), (2, None)] + [(0, C.byref(joint(**kw))) for kw in BAD_JOINTS])
    base = [C.byref(j), 4, FAKE, 8, FAKE, 8, FAKE, 8, FAKE, 8, FAKE, 1, FAKE, FAKE, None, FAKE, FAKE, 8, FAKE, 8, FAKE, 1,
            FAKE, FAKE, FAKE, None, FAKE, FAKE, need.value, None]
    refuse(base, lib.abcd_residual_norm_bwd,
           [(0, None), (1, -1), (2, None), (2, FAKE + 1), (3, 7), (4, FAKE + 1), (5, 7), (6, None), (7, 7), (8, None),
            (9, 7), (10, None), (11, 0), (12, None), (13, None), (15, None), (15, FAKE + 2), (16, FAKE + 1), (17, 7),
            (18, FAKE + 1), (19, 7), (20, FAKE + 1), (21, 0), (22, FAKE + 1), (25, FAKE), (26, FAKE + 1), (27, None),
            (27, FAKE + 8), (28, need.value - 1)])
    refuse(base, lib.abcd_residual_norm_bwd, [(0, C.byref(joint(**kw))) for kw in BAD_JOINTS])
    base[0] = C.byref(joint(pre=0, pre_weight=None))
    refuse(base, lib.abcd_residual_norm_bwd, [(24, FAKE)])
    base[2], base[24] = None, None
    refuse(base, lib.abcd_residual_norm_bwd, [(4, None)])


@pytest.mark.parametrize("post,pre,gate", [("layer", "layer", "row"), ("rms", "rms", "full"), (None, "layer", "none"),
                                           ("rms", None, "row"), (None, "rms", "full"), ("layer", None, "none")])
def test_reference_joint_gradient_is_its_forwards(post, pre, gate):
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=D.F64).requires_grad_()
    n, d = 5, 9
    f, x = rand(n, d), rand(n, d)
    p = {k: rand(d) for k in ("post_weight", "post_bias", "pre_weight", "pre_bias", "scale")
         if not (k.startswith("post") and post is None) and not (k.startswith("pre") and pre is None)
         and not (k == "post_bias" and post == "rms") and not (k == "pre_bias" and pre == "rms")}
    gt = dict(none=None, row=rand(n, 1), full=rand(n, d))[gate]
    r = R.residual_norm(f, x, post, pre, p, gt, 1e-5)
    dy, dz = rand(n, d).detach(), rand(n, d).detach() if pre else None
    loss = (r["y"][0] * dy).sum() + ((r["z"][0] * dz).sum() if pre else 0)
    leaves = dict(f=f, x=x, **p, **({"gate": gt} if gt is not None else {}))
    want = dict(zip(leaves, torch.autograd.grad(loss, list(leaves.values()))))
    det = lambda t: None if t is None else t.detach()
    stats = {k: det(r[k][0]) for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd") if k in r}
    got = R.residual_norm_bwd(dz, dy, det(f), det(r["y"][0]), stats, post, pre, {k: det(v) for k, v in p.items()}, det(gt))
    for k, v in want.items():
        assert torch.allclose(got[k][0], v, rtol=1e-9, atol=1e-11), k


def layer(**kw):
    from paper_2608_27735_amd import _lib
    l = dict(dtype=F16, act=3, i=8, o=5, w=FAKE, b=FAKE)
    l.update(kw)
    return _lib.abcd_layer(*l.values())


BAD_LAYERS = [dict(dtype=3), dict(act=5), dict(act=-1), dict(i=0), dict(i=65537), dict(o=0), dict(o=65537)]


def test_linear_refuses(lib):
    l, need = layer(), C.c_size_t(0)
    assert lib.abcd_linear_workspace_size(C.byref(l), 4, C.byref(need)) == 0 and need.value == 0  # of a few rows
    for size in (lib.abcd_linear_workspace_size, lib.abcd_linear_bwd_workspace_size):
        assert size(C.byref(layer(i=300)), 400, C.byref(need)) == 0 and need.value >= 400
        refuse([C.byref(l), 4, C.byref(need)], size,
               [(0, None), (1, -1), (1, (1 << 30) + 1), (2, None)] + [(0, C.byref(layer(**kw))) for kw in BAD_LAYERS])
    l = layer(i=300)
    lib.abcd_linear_workspace_size(C.byref(l), 400, C.byref(need))
    base = [C.byref(l), 400, FAKE, 300, FAKE, 5, FAKE, 5, FAKE, FAKE, need.value, None]
    bad = BAD_LAYERS + [dict(w=None), dict(w=FAKE + 1), dict(b=FAKE + 1)]
    refuse(base, lib.abcd_linear,
           [(0, C.byref(layer(**kw))) for kw in bad] +
           [(0, None), (1, -1), (2, None), (2, FAKE + 1), (3, 299), (4, FAKE + 1), (5, 4), (6, None), (7, 4), (8, FAKE + 8),
            (9, None), (9, FAKE + 16), (10, need.value - 1)])
    l = layer()
    lib.abcd_linear_bwd_workspace_size(C.byref(l), 400, C.byref(need))
    base = [C.byref(l), 400, FAKE, 5, FAKE, 8, None, None, FAKE, FAKE, 8, FAKE, FAKE, FAKE, need.value, None]
    refuse(base, lib.abcd_linear_bwd,
           [(0, C.byref(layer(**kw))) for kw in bad] +
           [(0, None), (1, -1), (2, None), (2, FAKE + 1), (3, 4), (4, None), (4, FAKE + 1), (5, 7), (6, FAKE), (7, FAKE),
            (8, FAKE + 8), (9, FAKE + 1), (10, 7), (11, FAKE + 1), (12, FAKE + 1), (13, None), (13, FAKE + 16),
            (14, need.value - 1)])
    base[4], base[6], base[7] = None, FAKE, FAKE
    refuse(base, lib.abcd_linear_bwd, [(4, FAKE), (6, FAKE + 8), (6, None), (7, None)])


def test_the_gated_block_refuses_a_layers_activations(lib):
    from paper_2608_27735_amd import _lib
    for a in (3, 4):
        f = _lib.abcd_ffn(F16, a, 8, 8, 8, FAKE, FAKE, FAKE, None, None, None, 0.0, 0, 0)
        assert lib.abcd_gated_ffn_workspace_size(C.byref(f), 4, 0, C.byref(C.c_size_t(0))) == 1


@pytest.mark.parametrize("name", [None, "silu", "gelu", "relu", "sigmoid"])
def test_reference_linear_gradient_is_its_forwards(name):
    g = torch.Generator().manual_seed(5)
    x, w, b, res, dy = (torch.randn(*s, generator=g, dtype=D.F64).requires_grad_()
                        for s in ((6, 4), (3, 4), (3,), (6, 3), (6, 3)))
    y, _ = R.linear(x, w, b, name, res)
    want = torch.autograd.grad((y * dy.detach()).sum(), (x, w, b))
    got = R.linear_bwd(*(t.detach() for t in (dy, x, w, b)), name, 0.0, 0.0)
    for k, v in zip(("x", "w", "b"), want):
        assert torch.allclose(got[k][0], v, rtol=1e-9, atol=1e-11), k
