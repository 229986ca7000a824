"""A linear layer from solved codes to serving: the descent, the norm, the 8-bit products and their gradients together.

    python examples/quantised_layer.py            (needs an MI355X and the built library)

1. Hidden states go through a layer norm; its result X and full-precision weights W give the outputs the layer should have.
2. dmmv_solve finds 4-bit codes for every row of W that keep the largest output error down.
3. The codes are a block matrix with a scale per row.  They stay fixed; the norm's gamma and beta and the layer's bias are
   trained towards outputs of another norm and bias, as a layer is adapted to a task.  What the backward pass keeps of a
   step is in 8 bits: the checkpoint of the hidden states and the product's operand.
4. The same from 8-bit weights that are trained themselves, with the gradient of the weights from the checkpoint.
5. One token through the trained layer.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2508_13437_amd import dmmv


def hidden_states(tokens, features, g):
    x = torch.randn(tokens, features, generator=g) * torch.exp(0.5 * torch.randn(tokens, 1, generator=g))
    x[:, torch.randperm(features, generator=g)[:max(1, features // 100)]] *= 20.0
    return x.to(torch.bfloat16)


def solve_codes(X, W, bits=4, iters=50):
    """4-bit codes [rows][features] (float32 integers) and scales [rows] for X W^T, by the pruned descent."""
    half = 2 ** (bits - 1)
    scale = W.abs().amax(1) / (half - 1)
    x0 = torch.round(W / scale[:, None]).clamp(-half, half - 1)
    D = np.arange(-half, half, dtype=np.float32)
    with dmmv.Handle(A=X.t().contiguous().t(), b=(W @ X.t()).contiguous(), D=D, scale=scale.cpu().numpy(), prune=True) as h:
        before = (x0 * scale[:, None] @ X.t() - W @ X.t()).abs().amax(1)
        res = dmmv.dmmv_solve(h, x0, iters)
    return res.x, scale, before, res.max_violation


class Layer:
    """norm -> 8 bits -> product + bias; forward keeps 8-bit checkpoints, backward reads them."""

    def __init__(self, gamma, beta, bias, w):
        self.gamma, self.beta, self.bias, self.w = gamma, beta, bias, w

    def forward(self, h):
        n = dmmv.dmmv_layernorm(h, self.gamma, self.beta, y=False, q=True, xq=True)
        self.kept = n
        return dmmv.dmmv_block_product(n.q, self.w, self.bias)

    def backward(self, dy, weights=False):
        n = self.kept
        dx, dw, dbias = dmmv.dmmv_block_backward(dy, n.q, self.w, dw=weights)
        dh, dgamma, dbeta = dmmv.dmmv_layernorm_backward(dx, n.xq, self.gamma, n.mean, n.rstd)
        return dh, dgamma, dbeta, dbias, dw


def train(layer, h, target, steps, lr, weights=None):
    """Adam on the squared error.  weights: float32 master copy of 8-bit weights, quantised again after every step."""
    params = [layer.gamma, layer.beta, layer.bias] + ([weights] if weights is not None else [])
    opt = torch.optim.Adam([p.requires_grad_() for p in params], lr=lr)
    losses = []
    for _ in range(steps):
        with torch.no_grad():
            if weights is not None:
                layer.w = dmmv.dmmv_block_quantize(weights, 128)
            diff = layer.forward(h).float() - target
            losses.append(float(diff.square().mean()))
            _, dgamma, dbeta, dbias, dw = layer.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16), weights is not None)
            for p, g in zip(params, (dgamma, dbeta, dbias, dw)):
                p.grad = g
        opt.step()
    for p in params:
        p.requires_grad_(False)
    return losses


def run(tokens=512, features=256, rows=384, steps=60, device="cuda:0", seed=1):
    g = torch.Generator().manual_seed(seed)
    h = hidden_states(tokens, features, g).to(device)
    W = (torch.randn(rows, features, generator=g) * 0.02).to(device)
    gamma0 = (1.0 + 0.1 * torch.randn(features, generator=g)).to(device)
    beta0 = (0.1 * torch.randn(features, generator=g)).to(device)
    X = dmmv.dmmv_layernorm(h.float(), gamma0, beta0).y
    target = X @ W.t()

    codes, scale, before, after = solve_codes(X, W)
    solved = dmmv.BlockMatrix(codes.to(torch.float8_e4m3fn), scale[:, None].expand(rows, -(-features // 128)))
    task = dmmv.dmmv_layernorm(h.float(), gamma0 + (0.3 * torch.randn(features, generator=g)).to(device), -beta0).y @ W.t()
    layer = Layer(gamma0.clone(), beta0.clone(), torch.zeros(rows, device=device), solved)
    frozen = train(layer, h, task + 0.1, steps, 2e-2)

    master = torch.randn(rows, features, generator=g).to(device) * 0.02
    other = Layer(gamma0.clone(), beta0.clone(), torch.zeros(rows, device=device), None)
    trained = train(other, h, target, steps, 2e-3, master)

    batch = layer.forward(h)
    token = layer.forward(h[:1])
    return dict(rounded=float(before.max()), solved=float(after.max()), frozen=frozen, trained=trained, batch=batch, token=token)


if __name__ == "__main__":
    r = run()
    print(f"largest output error: {r['rounded']:.4f} by rounding, {r['solved']:.4f} solved")
    print(f"mean squared error, norm and bias adapted around the solved codes: {r['frozen'][0]:.3e} -> {r['frozen'][-1]:.3e}")
    print(f"mean squared error, 8-bit weights trained from random ones: {r['trained'][0]:.3e} -> {r['trained'][-1]:.3e}")
    print(f"one token: {r['token'][0, :4].tolist()}")
