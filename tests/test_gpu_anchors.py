"""The decoder of colours from shared features, which runs the operators around a
decoder's blocks together: its gradients against differences of a float64 evaluation
of the same formulas, its 8-bit checkpoints, training through the active-block step,
and its passes on another stream and replayed from a graph."""
import numpy as np
import pytest
import torch

import decoder_ref as D
import features_ref as R
from paper_2608_27735_amd import synthetic as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anchors():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_27735_amd import anchors
    return anchors


def make(anchors, n=70, m=11, **kw):
    index = torch.randint(0, m, (n,), generator=torch.Generator().manual_seed(n)).cuda()
    index[3] = -1  # a Gaussian without an anchor
    kw = dict(dict(feature_width=12, width=20, hidden=28, sh_degree=1, seed=4), **kw)
    dec = anchors.AnchorDecoder(index, m, **kw)
    # norms, gates and scales other than they start
    g = torch.Generator().manual_seed(9)
    for k, t in dec.weights.items():
        if not k.startswith("w_"):
            t.add_(0.2 * torch.randn(t.shape, generator=g).cuda())
    return dec


def forward64(dec, features, w):
    e = R.embed(features, dec.index.cpu(), dec.scale)
    x = R.act(e @ w["w_in"].T + w["b_in"], dec.act)[0]
    gate = R.act(x @ w["w_gate"].T + w["b_gate"], "sigmoid")[0]
    n = D.layer_norm(x, w["norm_weight"], w["norm_bias"], 1e-5)[0]
    f = D.ffn(n, {k: w[k[:2] + "block_" + k[2:]] for k in ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down")}, dec.act, 0.0)["y"][0]
    z = R.residual_norm(f, x, "layer", "layer", w, gate, 1e-5)["z"][0]
    return z @ w["w_out"].T + w["b_out"]


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradients_against_differences(anchors, act):
    dec = make(anchors, dtype=torch.float32, act=act)
    gen = torch.Generator().manual_seed(7)
    d_sh = torch.randn(70, 4, 3, generator=gen)
    x, w = D.d64(dec.features), {k: D.d64(v) for k, v in dec.weights.items()}
    ref = forward64(dec, x, w)
    assert (D.d64(dec.forward()).view(70, -1) - ref).abs().max() <= 1e-4 * ref.abs().max()
    g = dec.backward(d_sh.cuda())
    loss = lambda x, w: (forward64(dec, x, w) * d_sh.double().view(70, -1)).sum().item()
    gw = dec._views(g["weights"])
    # along random directions of all leaves together, and of each by itself
    leaves = [None, "features"] + list(w)
    for leaf in leaves:
        vx = torch.randn(x.shape, generator=gen, dtype=D.F64) * (leaf in (None, "features"))
        vw = {k: torch.randn(v.shape, generator=gen, dtype=D.F64) * (leaf in (None, k)) for k, v in w.items()}
        e = 1e-5
        diff = (loss(x + e * vx, {k: w[k] + e * vw[k] for k in w}) -
                loss(x - e * vx, {k: w[k] - e * vw[k] for k in w})) / (2 * e)
        terms = [D.d64(g["features"]) * vx] + [D.d64(gw[k]) * vw[k] for k in w]
        along, size = sum(t.sum().item() for t in terms), sum(t.abs().sum().item() for t in terms)
        assert abs(diff - along) <= 2e-5 * size, (leaf, diff, along)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_checkpoints_stand_for_what_they_keep(anchors, dtype, monkeypatch):
    """With 8-bit checkpoints the backward pass is that of the numbers they hold."""
    d_sh = torch.randn(70, 4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    a, b, c = (make(anchors, dtype=dtype, checkpoints8=k) for k in (True, True, False))
    sh = a.forward()
    got = a.backward(d_sh)
    pack8 = anchors.api.pack8
    monkeypatch.setattr(anchors.api, "pack8", lambda x: anchors.api.unpack8(pack8(x)))
    assert torch.equal(b.forward(), sh) and torch.equal(c.forward(), sh)
    want = b.backward(d_sh)
    assert all(torch.equal(got[k], want[k]) for k in want)
    plain = c.backward(d_sh)
    assert not torch.equal(plain["weights"], got["weights"])  # they were used


def test_it_trains_through_the_step(anchors):
    from paper_2608_27735_amd.train import NAMES, render_joint
    w = S.ring(n=2048, width=64, height=64, n_cams=3)
    params = {k: torch.from_numpy(np.ascontiguousarray(w.scene[k])).cuda() for k in NAMES}
    stored = params["sh"].clone()
    targets = [render_joint(c, w.params, params)[..., :3].contiguous() for c in w.cams]
    index = (torch.arange(2048, device="cuda") % 700).int()
    dec = anchors.AnchorDecoder(index, 700, sh_degree=w.params.sh_degree, checkpoints8=True, seed=1)
    before = dec.features.clone(), dec.flat.clone()
    losses = anchors.fit(w.cams, targets, w.params, params, dec, 6)
    assert len(losses) == 6 and all(np.isfinite(losses))
    assert torch.isfinite(dec.flat).all() and torch.isfinite(dec.features).all()
    assert not torch.equal(dec.features, before[0]) and not torch.equal(dec.flat, before[1])
    assert torch.equal(params["sh"], stored)  # the caller's parameters are not written


def test_a_forward_without_training_keeps_what_training_needs(anchors):
    d_sh = torch.randn(70, 4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    a, b = make(anchors), make(anchors)
    with pytest.raises(ValueError):
        a.backward(d_sh)
    want, got = a.forward(), b.forward()
    b.forward(train=False)
    assert torch.equal(want, got)
    want, got = a.backward(d_sh), b.backward(d_sh)
    assert all(torch.equal(want[k], got[k]) for k in want)
    with pytest.raises(ValueError):
        a.backward(d_sh)


@pytest.mark.parametrize("n,m,width", [(70, 11, 20), (9000, 300, 64), (9000, 300, 100)])
def test_on_another_stream_and_from_a_graph(anchors, n, m, width):
    """The same results on a stream of its own, beside other work, and on every replay of a
    captured step, whose inputs change between replays; two captured steps of two decoders
    keep to their own memory."""
    gen = torch.Generator().manual_seed(3)
    d = [torch.randn(n, 4, 3, generator=gen).cuda() for _ in range(4)]
    decs = [make(anchors, n, m, width=width, checkpoints8=k == 1) for k in range(2)]

    def step(dec, d_sh):
        sh = dec.forward()
        g = dec.backward(d_sh)
        return sh, g["features"].clone(), g["weights"].clone()

    want = [[step(dec, v) for v in d] for dec in decs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    busy = torch.randn(1024, 1024, device="cuda")
    with torch.cuda.stream(side):
        got = [step(decs[0], v) for v in d]
    for _ in range(4):
        busy = busy @ busy * 1e-3
    here = [step(decs[1], v) for v in d]
    torch.cuda.synchronize()
    for a, b in zip(got + here, want[0] + want[1]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    graphs, ins, outs = [], [], []
    for dec in decs:
        x = d[0].clone()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step(dec, x)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(dec, x)
        graphs.append(g), ins.append(x), outs.append(out)
    for k in (1, 2, 3, 0, 2):
        for x in ins:
            x.copy_(d[k])
        for g in graphs:
            g.replay()
        eager = step(decs[0], d[k])  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want[0][k]))
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i][k])), (k, i)


def test_checkpoints_take_less_memory(anchors):
    """What a forward keeps for training: with 8-bit checkpoints the rows of features and the
    last layer's input lie in 8 bits and an exponent for 32, and nothing is kept beside that."""
    n, fw, width = 1000, 48, 80

    def kept(checkpoints8):
        dec = make(anchors, n, 11, feature_width=fw, width=width, checkpoints8=checkpoints8)
        dec.forward()
        found, todo = {}, [dec._kept]
        while todo:
            v = todo.pop()
            if isinstance(v, torch.Tensor):
                s = v.untyped_storage()
                found[s.data_ptr()] = s.nbytes()
            elif isinstance(v, dict):
                todo += v.values()
            elif isinstance(v, (list, tuple)):
                todo += v
        return sum(found.values())

    bits16, bits8 = 2 * (fw + width) * n, sum(33 * ((d + 31) // 32) for d in (fw, width)) * n
    assert kept(False) - kept(True) == bits16 - bits8


def test_only_what_a_checkpoint_holds_is_rounded(anchors):
    """The gate's weights have the gradient of x itself, which is there in full."""
    d_sh = torch.randn(70, 4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    a, b = (make(anchors, checkpoints8=k) for k in (True, False))
    got, want = ({k: v.clone() for k, v in dec._views(dec.backward(d_sh)["weights"]).items()} for dec in (a, b)
                 if dec.forward() is not None)
    assert all(torch.equal(got[k], want[k]) for k in want if k not in ("w_in", "b_in", "w_out"))
    assert not torch.equal(got["w_out"], want["w_out"])  # z is one of the checkpoints


def test_decoder_of_no_gaussians(anchors):
    dec = anchors.AnchorDecoder(torch.zeros(0, dtype=torch.int32, device="cuda"), 5, feature_width=12, width=20, hidden=28, sh_degree=1)
    sh = dec.forward()
    assert sh.shape == (0, 4, 3)
    g = dec.backward(sh)
    assert all((v == 0).all() for v in g.values())


def test_anchors_are_those_at_construction(anchors):
    """A caller's later change of index reaches neither the lookup nor the gradient's sort."""
    d_sh = torch.randn(70, 4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    index = (torch.arange(70) * 3 % 11).cuda()
    kw = dict(feature_width=12, width=20, hidden=28, sh_degree=1, seed=4)
    a, b = (anchors.AnchorDecoder(i, 11, **kw) for i in (index, index.clone()))
    index.fill_(0)
    assert torch.equal(a.forward(), b.forward())
    got, want = a.backward(d_sh), b.backward(d_sh)
    assert all(torch.equal(got[k], want[k]) for k in want)
