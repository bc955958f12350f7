"""Colours of the active block from learned features instead of stored ones: a
decoder of two pre-norm gated feed-forward blocks, trained through the
active-block step.

Every Gaussian has a feature row x. The decoder makes
    y  = x + dropout(ffn1(layer_norm1(x)))
    sh = ffn2(layer_norm2(y))
and the step renders with these SH coefficients, so that their gradient
(abcd_render_bwd's d_sh) is the decoder's upstream one. Features and weights
are kept in fp32 for Adam; the operators run in `dtype`. Run as a program it
fits the colours of a small synthetic scene from random features:
    python -m paper_2608_27735_amd.decoder
"""
import torch

from . import api
from .step import ActiveBlockStep
from .train import NAMES, psnr, render_joint


class FeatureDecoder:
    """Forward and backward pass of the decoder for n Gaussians, and its Adam
    update. features: [n, width] in fp32 (random if not given)."""

    def __init__(self, n, width=64, hidden=128, sh_degree=3, features=None, dtype=torch.bfloat16,
                 p=0.0, act="silu", seed=0, device=None):
        dev = device or torch.device("cuda", torch.cuda.current_device())
        self.dtype, self.p, self.act, self.seed, self.calls = dtype, float(p), act, int(seed), 0
        self.nc = (sh_degree + 1) ** 2
        out = 3 * self.nc
        g = torch.Generator(device=dev)
        g.manual_seed(self.seed)
        shapes = dict(norm1_weight=(width,), norm1_bias=(width,), norm2_weight=(width,),
                      norm2_bias=(width,))
        for i, o in ((1, width), (2, out)):
            shapes.update({f"w_gate{i}": (hidden, width), f"w_up{i}": (hidden, width),
                           f"w_down{i}": (o, hidden), f"b_gate{i}": (hidden,),
                           f"b_up{i}": (hidden,), f"b_down{i}": (o,)})
        # one flat array of every weight, and views into it: one group for Adam,
        # one conversion for the operators
        self.shapes = shapes
        total = sum(torch.Size(s).numel() for s in shapes.values())
        self.flat = torch.zeros(total, device=dev)
        self.weights = self._views(self.flat)
        for k, t in self.weights.items():
            if k.startswith("w_"):
                t.copy_(torch.randn(t.shape, generator=g, device=dev) * t.shape[1] ** -0.5)
            elif k.endswith("weight"):
                t.fill_(1.0)
        if features is None:
            features = torch.randn((n, width), generator=g, device=dev)
        self.features = features.to(device=dev, dtype=torch.float32).contiguous()
        if self.features.shape != (n, width):
            raise ValueError(f"features must have shape ({n}, {width})")
        self.params = dict(features=self.features, weights=self.flat)
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self._grad = self._views(self.grads["weights"])
        self.m = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.v = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.t = 0
        self._kept = None

    def _views(self, flat):
        views, at = {}, 0
        for k, s in self.shapes.items():
            size = torch.Size(s).numel()
            views[k] = flat[at:at + size].view(s)
            at += size
        return views

    def _ffn(self, w, i):
        """Block i's weights; contiguous by themselves."""
        return {k: w[f"{k}{i}"] for k in api.FFN_WEIGHTS + api.FFN_BIASES}

    def forward(self, train=True):
        """SH coefficients [n, (sh_degree + 1)^2, 3] in fp32. train: dropout, and
        what backward() needs is kept; every such call has a mask of its own."""
        w = self._views(self.flat.to(self.dtype))
        x = self.features.to(self.dtype)
        p = self.p if train else 0.0
        offset = self.calls
        self.calls += 1 if train else 0
        n1 = api.layer_norm(x, w["norm1_weight"], w["norm1_bias"])
        f1 = api.gated_ffn(n1["y"], self._ffn(w, 1), self.act, residual=x, p=p, seed=self.seed,
                           offset=offset, save=train)
        n2 = api.layer_norm(f1["y"], w["norm2_weight"], w["norm2_bias"])
        f2 = api.gated_ffn(n2["y"], self._ffn(w, 2), self.act, save=train)
        if train:
            self._kept = (w, x, n1, f1, n2, f2, p, offset)
        return f2["y"].float().view(-1, self.nc, 3)

    def backward(self, d_sh):
        """Gradients of features and weights from the gradient of the SH coefficients
        that the last forward() with train=True gave; once for each of these."""
        if self._kept is None:
            raise ValueError("backward() needs a forward() with train=True before it")
        w, x, n1, f1, n2, f2, p, offset = self._kept
        self._kept = None
        d = d_sh.reshape(x.shape[0], -1).to(self.dtype)
        g2 = api.gated_ffn_bwd(d, n2["y"], self._ffn(w, 2), self.act, saved=f2["saved"])
        d2 = api.layer_norm_bwd(g2["x"], f1["y"], n2["mean"], n2["rstd"], w["norm2_weight"])
        # f1's gradient reaches x by the residual path and through the block
        g1 = api.gated_ffn_bwd(d2["x"], n1["y"], self._ffn(w, 1), self.act, saved=f1["saved"], p=p,
                               seed=self.seed, offset=offset)
        d1 = api.layer_norm_bwd(g1["x"], x, n1["mean"], n1["rstd"], w["norm1_weight"], add=d2["x"])
        self.grads["features"].copy_(d1["x"])
        for i, g, norm in ((1, g1, d1), (2, g2, d2)):
            for k in api.FFN_WEIGHTS + api.FFN_BIASES:
                self._grad[f"{k}{i}"].copy_(g[k])
            self._grad[f"norm{i}_weight"].copy_(norm["weight"])
            self._grad[f"norm{i}_bias"].copy_(norm["bias"])
        return self.grads

    def update(self, lr):
        """One Adam update of features and weights."""
        self.t += 1
        api.adam_step(self.params, self.grads, self.m, self.v, lr, self.t)


def fit(cams, targets, prm, params, decoder, steps, lr=2e-3, rng=None):
    """`steps` training steps of the decoder over the cameras in turn, everything
    but the colours fixed: the active-block step with the decoder's SH
    coefficients in place of stored ones. params: the block's parameters (their sh
    is not read). Returns the loss of every step."""
    params = dict(params)
    params["sh"] = decoder.forward(train=False).contiguous()
    st = ActiveBlockStep(cams[0], prm, params)
    losses = []
    for i in range(steps):
        c = i % len(cams) if rng is None else int(rng.integers(len(cams)))
        params["sh"].copy_(decoder.forward())
        st.cam = cams[c]
        st.loss.zero_()
        st.project_and_bin(sync=True)
        st.forward()
        st.loss_grad(targets[c])
        st.backward(st.dL_dout)
        decoder.backward(st.grads["sh"])
        decoder.update(lr)
        losses.append(st.loss.clone())
    return [float(v) for v in torch.stack(losses).cpu()[:, 0]] if losses else []


def main():
    from . import synthetic
    w = synthetic.ring(n=8192, width=128, height=128, n_cams=4)
    params = {k: torch.from_numpy(w.scene[k]).cuda() for k in NAMES}
    targets = [render_joint(c, w.params, params)[..., :3].contiguous() for c in w.cams]
    dec = FeatureDecoder(len(w.scene["means"]), sh_degree=w.params.sh_degree, p=0.05, seed=1)

    def score():
        shown = dict(params, sh=dec.forward(train=False).contiguous())
        return sum(psnr(render_joint(c, w.params, shown), t)
                   for c, t in zip(w.cams, targets)) / len(targets)

    before = score()
    losses = fit(w.cams, targets, w.params, params, dec, 200)
    print(f"L1 loss {losses[0]:.4f} -> {losses[-1]:.4f}, PSNR {before:.2f} -> {score():.2f} dB")


if __name__ == "__main__":
    main()
