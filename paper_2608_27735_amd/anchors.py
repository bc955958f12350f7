"""Colours of the active block decoded from features that Gaussians share.

A scene has fewer anchors than Gaussians; every Gaussian has an anchor's index and
takes its feature row. The decoder makes, with block = ffn(norm) of a gated
feed-forward block,
    x = silu(scale features[index] w_in' + b_in)
    g = sigmoid(x w_gate' + b_gate)
    y = x + s g layer_norm(ffn(layer_norm(x))),  z = layer_norm(y)
    sh = z w_out' + b_out
and the step renders with these SH coefficients. Features and weights are kept in
fp32 for Adam; the operators run in `dtype`. With checkpoints8 the first and the last
linear layer's inputs are kept for the backward pass in 8 bits (x itself, the gate's
input, is needed there by the norm and kept as it is). Run as a program it fits the
colours of a small synthetic scene:
    python -m paper_2608_27735_amd.anchors
"""
import torch

from . import api
from .decoder import fit
from .train import NAMES, psnr, render_joint


class AnchorDecoder:
    """Forward and backward pass of the decoder and its Adam update, for Gaussians
    whose anchors are index [n] (int32 or int64). features: [m, feature_width] in
    fp32 (random if not given)."""

    def __init__(self, index, m, feature_width=32, width=64, hidden=128, sh_degree=3, features=None,
                 dtype=torch.bfloat16, act="silu", checkpoints8=False, seed=0):
        dev = index.device
        # a copy: what embed_sort makes of it below belongs to these anchors
        self.index, self.m, self.dtype, self.act = index.clone(), int(m), dtype, act
        self.checkpoints8 = bool(checkpoints8)
        self.scale = float(feature_width) ** 0.5
        self.nc = (sh_degree + 1) ** 2
        out = 3 * self.nc
        g = torch.Generator(device=dev)
        g.manual_seed(int(seed))
        self.shapes = dict(
            w_in=(width, feature_width), b_in=(width,), w_block_gate=(hidden, width),
            b_block_gate=(hidden,), w_block_up=(hidden, width), b_block_up=(hidden,),
            w_block_down=(width, hidden), b_block_down=(width,), w_gate=(width, width), b_gate=(width,),
            w_out=(out, width), b_out=(out,), norm_weight=(width,), norm_bias=(width,), post_weight=(width,),
            post_bias=(width,), pre_weight=(width,), pre_bias=(width,), scale=(width,))
        # one flat array of every weight, and views into it: one group for Adam,
        # one conversion for the operators
        total = sum(torch.Size(s).numel() for s in self.shapes.values())
        self.flat = torch.zeros(total, device=dev)
        self.weights = self._views(self.flat)
        for k, t in self.weights.items():
            if k.startswith("w_"):
                t.copy_(torch.randn(t.shape, generator=g, device=dev) * t.shape[1] ** -0.5)
            elif k.endswith("weight"):
                t.fill_(1.0)
            elif k == "scale":
                t.fill_(0.5)
        if features is None:
            features = torch.randn((self.m, feature_width), generator=g, device=dev) * feature_width ** -0.5
        self.features = features.to(device=dev, dtype=torch.float32).contiguous()
        if self.features.shape != (self.m, feature_width):
            raise ValueError(f"features must have shape ({self.m}, {feature_width})")
        # anchors do not change: their positions are sorted once for all steps
        self.sorted = api.embed_sort(self.index, self.m)
        self.params = dict(features=self.features, weights=self.flat)
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self._grad = self._views(self.grads["weights"])
        self.m1 = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.m2 = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.t = 0
        self._kept = None

    def _views(self, flat):
        views, at = {}, 0
        for k, s in self.shapes.items():
            size = torch.Size(s).numel()
            views[k] = flat[at:at + size].view(s)
            at += size
        return views

    @staticmethod
    def _ffn(w):
        return dict(w_gate=w["w_block_gate"], b_gate=w["b_block_gate"], w_up=w["w_block_up"], b_up=w["b_block_up"],
                    w_down=w["w_block_down"], b_down=w["b_block_down"])

    @staticmethod
    def _joint(w):
        return dict(post="layer", pre="layer", params={k: w[k] for k in api.JOINT_PARAMS})

    def forward(self, train=True):
        """SH coefficients [n, (sh_degree + 1)^2, 3] in fp32. train: what backward()
        needs is kept."""
        w = {k: v.contiguous() for k, v in self._views(self.flat.to(self.dtype)).items()}
        keep = api.pack8 if self.checkpoints8 else (lambda t: t)
        e = api.embed(self.features, self.index, self.scale, dtype=self.dtype)
        x = api.linear(e, w["w_in"], w["b_in"], self.act)["y"]
        gate = api.linear(x, w["w_gate"], w["b_gate"], "sigmoid")["y"]
        n = api.layer_norm(x, w["norm_weight"], w["norm_bias"])
        f = api.gated_ffn(n["y"], self._ffn(w), self.act, save=train)
        j = api.residual_norm(f["y"], x, gate=gate, **self._joint(w))
        sh = api.linear(j["z"], w["w_out"], w["b_out"])["y"]
        if train:
            z = keep(j.pop("z"))  # all that the backward pass needs of j are y and the statistics
            self._kept = (w, keep(e), x, gate, n, f, j, z)
        return sh.float().view(len(self.index), self.nc, 3)

    def backward(self, d_sh):
        """Gradients of features and weights from the gradient of the SH coefficients
        that the last forward() with train=True gave; once for each of these."""
        if self._kept is None:
            raise ValueError("backward() needs a forward() with train=True before it")
        w, e, x, gate, n, f, j, z = self._kept
        self._kept = None
        d = d_sh.reshape(len(self.index), 3 * self.nc).to(self.dtype)
        out = api.linear_bwd(d, z, w["w_out"], w["b_out"])
        gj = api.residual_norm_bwd(out["x"], None, f["y"], j, gate=gate, **self._joint(w))
        # x's gradient comes by the residual path, through the gate and through the block
        gg = api.linear_bwd(gj["gate"], x, w["w_gate"], w["b_gate"], "sigmoid")
        gf = api.gated_ffn_bwd(gj["f"], n["y"], self._ffn(w), self.act, saved=f["saved"])
        gn = api.layer_norm_bwd(gf["x"], x, n["mean"], n["rstd"], w["norm_weight"], add=gj["x"])
        dx = gn["x"].add_(gg["x"])
        gi = api.linear_bwd(dx, e, w["w_in"], w["b_in"], self.act)
        api.embed_bwd(gi["x"], self.sorted, self.m, self.scale, out=self.grads["features"])
        for names, grads in ((("w_out", "b_out"), out), (("w_gate", "b_gate"), gg), (("w_in", "b_in"), gi)):
            for k in names:
                self._grad[k].copy_(grads[k[0]])
        for k in api.FFN_WEIGHTS + api.FFN_BIASES:
            self._grad[k[:2] + "block_" + k[2:]].copy_(gf[k])
        for k in api.JOINT_PARAMS:
            self._grad[k].copy_(gj[k])
        self._grad["norm_weight"].copy_(gn["weight"])
        self._grad["norm_bias"].copy_(gn["bias"])
        return self.grads

    def update(self, lr):
        """One Adam update of features and weights."""
        self.t += 1
        api.adam_step(self.params, self.grads, self.m1, self.m2, lr, self.t)


def main():
    from . import synthetic
    w = synthetic.ring(n=8192, width=128, height=128, n_cams=4)
    params = {k: torch.from_numpy(w.scene[k]).cuda() for k in NAMES}
    targets = [render_joint(c, w.params, params)[..., :3].contiguous() for c in w.cams]
    n, m = len(w.scene["means"]), 2048
    # Gaussians next to each other along x share an anchor
    order = params["means"][:, 0].argsort()
    index = torch.empty(n, dtype=torch.int32, device="cuda")
    index[order] = (torch.arange(n, device="cuda") * m // n).int()
    dec = AnchorDecoder(index, m, sh_degree=w.params.sh_degree, checkpoints8=True, seed=1)

    def score():
        shown = dict(params, sh=dec.forward(train=False).contiguous())
        return sum(psnr(render_joint(c, w.params, shown), t)
                   for c, t in zip(w.cams, targets)) / len(targets)

    before = score()
    losses = fit(w.cams, targets, w.params, params, dec, 200)
    print(f"L1 loss {losses[0]:.4f} -> {losses[-1]:.4f}, PSNR {before:.2f} -> {score():.2f} dB")


if __name__ == "__main__":
    main()
