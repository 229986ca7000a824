"""Two residual blocks around quantised layers, trained and served: products with their activation, norms with gate and residual scale, clipped
gradients.

    python examples/quantised_block.py            (needs an MI355X and the built library)

The first block has a norm on both sides, a gate per channel and a residual scale; the second adds its input in the epilogue of its last product.
Activations that a product reads are in 8 bits and never exist otherwise; weights are 32-bit master copies, quantised again after every step.
1. The blocks learn the outputs of another pair of blocks with full-precision weights, by Adam on clipped gradients.
2. One token through the trained blocks.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2508_13437_amd import dmmv

ALPHA = 0.9
WEIGHTS, VECTORS = ("w1", "w2", "w3", "w4"), ("b1", "b2", "b3", "b4", "gamma", "beta", "post_gamma", "pre_gamma", "gate")


def parameters(features, hidden, g, device="cuda:0"):
    """Weights [out][in] and vectors of two blocks features -> hidden -> features, in 32 bits."""
    new = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    p = {"w1": new(hidden, features), "w2": new(features, hidden), "w3": new(hidden, features), "w4": new(features, hidden)}
    p = {k: v / v.shape[1] ** 0.5 for k, v in p.items()}
    p.update(b1=0.1 * new(hidden), b2=0.1 * new(features), b3=0.1 * new(hidden), b4=0.1 * new(features), gamma=1 + 0.1 * new(features),
             beta=0.1 * new(features), post_gamma=1 + 0.1 * new(features), pre_gamma=1 + 0.1 * new(features), gate=0.5 + 0.1 * new(features))
    return {k: v.to(device) for k, v in p.items()}


class Blocks:
    """norm -> w1, act -> w2 -> post norm, gate, alpha -> norm -> w3, act -> w4 + residual."""

    def __init__(self, p, act="gelu", dtype=torch.bfloat16):
        self.p, self.act, self.dtype = p, act, dtype
        self.post, self.pre = dmmv.Norm(p["post_gamma"], rms=True), dmmv.Norm(p["pre_gamma"], rms=True)
        self.quantise()

    def quantise(self):
        self.w = {k: dmmv.dmmv_block_quantize(self.p[k], 128) for k in WEIGHTS}

    def forward(self, h):
        p, w, kind = self.p, self.w, self.dtype
        n = dmmv.dmmv_layernorm(h, p["gamma"], p["beta"], y=False, q=True)
        a = dmmv.dmmv_block_linear(n.q, w["w1"], p["b1"], self.act, dtype=kind, y=False, q=True, u=True)
        f = dmmv.dmmv_block_linear(a.q, w["w2"], p["b2"], dtype=kind).y
        s = dmmv.dmmv_residual_norm(f, h, self.post, self.pre, p["gate"], alpha=ALPHA, y=False, q=True)
        b = dmmv.dmmv_block_linear(s.q, w["w3"], p["b3"], self.act, dtype=kind, y=False, q=True, u=True)
        self.kept = h, n, a, f, s, b
        return dmmv.dmmv_block_linear(b.q, w["w4"], p["b4"], residual=s.h, dtype=kind).y

    def backward(self, dy):
        """The gradients by the parameters' names, and the input's."""
        p, w = self.p, self.w
        h, n, a, f, s, b = self.kept
        g = {}
        dx, g["w4"], g["b4"] = dmmv.dmmv_block_backward(dy, b.q, w["w4"])
        du, g["b3"] = dmmv.dmmv_activation_backward(dx, b.u, self.act)
        dn, g["w3"], _ = dmmv.dmmv_block_backward(du, s.q, w["w3"], dbias=False)
        r = dmmv.dmmv_residual_norm_backward(dn, dy, f, s, self.post, self.pre, p["gate"], alpha=ALPHA)
        g["gate"], g["post_gamma"], g["pre_gamma"] = r.dgate, r.dpost_gamma, r.dgamma
        dx, g["w2"], g["b2"] = dmmv.dmmv_block_backward(r.df, a.q, w["w2"])
        du, g["b1"] = dmmv.dmmv_activation_backward(dx, a.u, self.act)
        dn, g["w1"], _ = dmmv.dmmv_block_backward(du, n.q, w["w1"], dbias=False)
        dh, g["gamma"], g["beta"] = dmmv.dmmv_layernorm_backward(dn, h, p["gamma"], n.mean, n.rstd)
        return g, dh + r.dh


def train(blocks, h, target, steps, lr, max_norm):
    opt = torch.optim.Adam([blocks.p[k].requires_grad_() for k in (*WEIGHTS, *VECTORS)], lr=lr)
    losses, norms = [], []
    for _ in range(steps):
        with torch.no_grad():
            diff = blocks.forward(h).float() - target
            losses.append(diff.square().mean())
            g, _ = blocks.backward((diff * (2.0 / diff.numel())).to(blocks.dtype))
            norms.append(dmmv.dmmv_gradient_clip(list(g.values()), max_norm))
            for k, v in g.items():
                blocks.p[k].grad = v
        opt.step()
        with torch.no_grad():
            blocks.quantise()
    for k in (*WEIGHTS, *VECTORS):
        blocks.p[k].requires_grad_(False)
    return [float(v) for v in losses], [float(v) for v in norms]


def hidden_states(tokens, features, g):
    return (torch.randn(tokens, features, generator=g) * torch.exp(0.3 * torch.randn(tokens, 1, generator=g))).to(torch.bfloat16)


def reference(p, h, act=torch.nn.functional.gelu):
    """The same blocks in PyTorch operations with full-precision weights."""
    x = torch.nn.functional.layer_norm(h, h.shape[1:], p["gamma"], p["beta"])
    f = act(x @ p["w1"].t() + p["b1"]) @ p["w2"].t() + p["b2"]
    rms = lambda v: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-5)  # noqa: E731
    s = ALPHA * h + p["gate"] * rms(f) * p["post_gamma"]
    return act(rms(s) * p["pre_gamma"] @ p["w3"].t() + p["b3"]) @ p["w4"].t() + p["b4"] + s


def run(tokens=512, features=256, hidden=640, steps=80, device="cuda:0", seed=1):
    g = torch.Generator().manual_seed(seed)
    h = hidden_states(tokens, features, g).to(device)
    target = reference(parameters(features, hidden, g, device), h.float())
    blocks = Blocks(parameters(features, hidden, g, device))
    losses, norms = train(blocks, h, target, steps, 2e-3, 1.0)
    batch = blocks.forward(h)
    return dict(losses=losses, norms=norms, batch=batch, token=blocks.forward(h[:1]))


if __name__ == "__main__":
    r = run()
    print(f"mean squared error {r['losses'][0]:.3e} -> {r['losses'][-1]:.3e}, gradient norm {r['norms'][0]:.3f} -> {r['norms'][-1]:.3f}")
    print(f"one token: {r['token'][0, :4].tolist()}")
