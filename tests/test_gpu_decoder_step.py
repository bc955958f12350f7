"""The decoder of colours from features: its gradients against differences of a
float64 evaluation of the same formulas, and training through the active-block
step."""
import numpy as np
import pytest
import torch

import decoder_ref as R
from paper_2608_27735_amd import synthetic as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def decoder():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_27735_amd import decoder
    return decoder


def forward64(dec, x, w, keep, p):
    ffn = lambda y, i, **kw: R.ffn(y, {k: w[f"{k}{i}"] for k in ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down")},
                                   dec.act, 0.0, **kw)["y"][0]
    y = ffn(R.layer_norm(x, w["norm1_weight"], w["norm1_bias"], 1e-5)[0], 1, res=x, keep=keep, p=p)
    return ffn(R.layer_norm(y, w["norm2_weight"], w["norm2_bias"], 1e-5)[0], 2)


@pytest.mark.parametrize("n,p", [(40, 0.0), (33, 0.2)])
def test_decoder_gradients_against_differences(decoder, n, p):
    dec = decoder.FeatureDecoder(n, width=20, hidden=28, sh_degree=1, dtype=torch.float32, p=p, act="gelu", seed=4)
    gen = torch.Generator().manual_seed(7)
    d_sh = torch.randn(n, 4, 3, generator=gen)
    for _ in range(2):  # the second call's mask is another one
        offset = dec.calls
        sh = dec.forward()
        keep = R.keep_mask(n, 20, p, 4, offset)
        x, w = R.d64(dec.features), {k: R.d64(v) for k, v in dec.weights.items()}
        ref = forward64(dec, x, w, keep, p)
        assert (R.d64(sh).view(n, -1) - ref).abs().max() <= 1e-4 * ref.abs().max()
        g = dec.backward(d_sh.cuda())
        loss = lambda x, w: (forward64(dec, x, w, keep, p) * d_sh.double().view(n, -1)).sum().item()
        gw = dec._views(g["weights"])
        for _ in range(3):
            vx = torch.randn(x.shape, generator=gen, dtype=R.F64)
            vw = {k: torch.randn(v.shape, generator=gen, dtype=R.F64) for k, v in w.items()}
            e = 1e-5
            diff = (loss(x + e * vx, {k: w[k] + e * vw[k] for k in w}) -
                    loss(x - e * vx, {k: w[k] - e * vw[k] for k in w})) / (2 * e)
            terms = [R.d64(g["features"]) * vx] + [R.d64(gw[k]) * vw[k] for k in w]
            along, size = sum(t.sum().item() for t in terms), sum(t.abs().sum().item() for t in terms)
            assert abs(diff - along) <= 1e-5 * size, (diff, along)


def test_decoder_trains_through_the_step(decoder):
    from paper_2608_27735_amd.train import NAMES, render_joint
    w = S.ring(n=4096, width=96, height=96, n_cams=3)
    params = {k: torch.from_numpy(np.ascontiguousarray(w.scene[k])).cuda() for k in NAMES}
    stored = params["sh"].clone()
    targets = [render_joint(c, w.params, params)[..., :3].contiguous() for c in w.cams]
    dec = decoder.FeatureDecoder(4096, sh_degree=w.params.sh_degree, p=0.05, seed=1)
    losses = decoder.fit(w.cams, targets, w.params, params, dec, 90)
    first, last = np.mean(losses[:3]), np.mean(losses[-3:])
    print(f"  L1 loss {first:.4f} -> {last:.4f}")
    assert last < 0.5 * first
    assert torch.equal(params["sh"], stored)  # the caller's parameters are not written


def test_a_forward_without_training_keeps_what_training_needs(decoder):
    """A look at the colours between a training forward and its backward changes
    neither; a backward without a forward is refused."""
    d_sh = torch.randn(50, 4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    a, b = (decoder.FeatureDecoder(50, width=24, hidden=32, sh_degree=1, p=0.2, seed=3) for _ in range(2))
    with pytest.raises(ValueError):
        a.backward(d_sh)
    want, got = a.forward(), b.forward()
    b.forward(train=False)
    assert torch.equal(want, got)
    want, got = a.backward(d_sh), b.backward(d_sh)
    assert all(torch.equal(want[k], got[k]) for k in want)
    with pytest.raises(ValueError):
        a.backward(d_sh)
