"""A quantised linear layer as it is trained and served: what its operators compute, as timed cases.

Three operators that follow one another in a layer whose weights the library has solved for (or that
are trained in 8 bits): the layer norm that makes the layer's input, the 8-bit checkpoint of an
activation, and the product of two 8-bit matrices with a scale for each block of 128, each with its
backward pass.

A block matrix holds e4m3 codes [rows][cols] and scales [rows / g][cols / 128], g = 1 or 128 (both
divisions rounded up); it stands for code * scale.  Quantising takes the smallest power of two that is
at least (largest finite |x| of the block) / 448, not below 2^-126, and 1 for a block of zeros.

    own = False: the operators in elementary torch operations, 32 bits;  True: the library's kernels
    listed()            the cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU
    run(state)          one pass, its outputs whole
    work(case)          bytes and flops one pass cannot do without
    exact(case, seed)   the same outputs in 64 bits, from the definitions
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
WIDTH = {"bf16": 2, "f32": 4}


# --------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------
# op        norm (forward), norm_grad, save (and restore), product, backward
# T, F, O   tokens, features (the contraction of the product), outputs of the layer
# out       norm: "8bit" = only the 8-bit result, the product's operand (serving);
#                 "save" = the result in the input's type and an 8-bit checkpoint of the input
# from_8bit norm_grad: the norm's input comes from its checkpoint
# weights   "blocks" = e4m3 with a power of two per 128 x 128 block; "solved" = the library's answer,
#           integers of 4 bits and a scale per row; "f32" = any 32-bit scales on both sides
def listed():
    return [
        # serving: the norm in front of a layer of 4096 features, a single token
        dict(name="norm_token", op="norm", dtype="bf16", T=1, F=4096, out="8bit"),
        # training: a batch of 4096 tokens, the input kept in 8 bits for the backward pass
        dict(name="norm_save", op="norm", dtype="bf16", T=4096, F=4096, out="save"),
        # backward, odd sizes, 32 bits: latency and the reduction over few rows
        dict(name="norm_grad_ragged", op="norm_grad", dtype="f32", T=513, F=1003, from_8bit=False),
        # backward of a training batch from the 8-bit checkpoint
        dict(name="norm_grad", op="norm_grad", dtype="bf16", T=4096, F=4096, from_8bit=True),
        # a checkpoint of odd size in 32 bits, saved and restored
        dict(name="save_ragged", op="save", dtype="f32", T=1365, F=2731, restore=True),
        # the checkpoint of an MLP's hidden activations
        dict(name="save_layer", op="save", dtype="bf16", T=4096, F=11008, restore=False),
        # serving a single token through an MLP-shaped layer: the weights are read once
        dict(name="product_token", op="product", dtype="bf16", T=1, F=4096, O=11008, weights="blocks"),
        # a few requests at once through a layer the library has solved (4 bits, a scale per row)
        dict(name="product_requests", op="product", dtype="bf16", T=24, F=4096, O=4096, weights="solved"),
        # a short prompt through a layer of odd sizes with 32-bit scales per block
        dict(name="product_ragged", op="product", dtype="f32", T=500, F=2731, O=1777, weights="f32"),
        # an MLP-shaped layer over a whole batch
        dict(name="product_layer", op="product", dtype="bf16", T=4096, F=4096, O=11008, weights="blocks"),
        # gradients of a layer of odd sizes, 32-bit gradients
        dict(name="backward_ragged", op="backward", dtype="f32", T=777, F=1003, O=1365, weights="blocks", dw=True),
        # gradients of the MLP-shaped layer over a whole batch
        dict(name="backward_layer", op="backward", dtype="bf16", T=4096, F=4096, O=11008, weights="blocks", dw=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "save", "product", "product", "backward", "backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    T, F = _log_uniform(rng, 1, 4096), _log_uniform(rng, 64, 4096)
    if rng.random() < 0.4:                                # layers are mostly multiples of a block
        F = -(-F // 128) * 128
    if op == "norm":
        return dict(op=op, dtype=dtype, T=T, F=F, out=rng.choice(["8bit", "save"]))
    if op == "norm_grad":
        return dict(op=op, dtype=dtype, T=T, F=F, from_8bit=rng.random() < 0.5)
    if op == "save":
        return dict(op=op, dtype=dtype, T=T, F=_log_uniform(rng, 64, 11008), restore=rng.random() < 0.5)
    O = _log_uniform(rng, 64, 11008)
    if rng.random() < 0.4:
        O = -(-O // 128) * 128
    if op == "product":
        return dict(op=op, dtype=dtype, T=T, F=F, O=O, weights=rng.choice(["blocks", "solved", "f32"]))
    weights = rng.choice(["blocks", "blocks", "solved"])
    # a solved layer is frozen: the gradient only passes through it
    return dict(op=op, dtype=dtype, T=T, F=F, O=O, weights=weights, dw=weights == "blocks")


# --------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------
def _spread(scales, rows, cols, g):
    """[rows][cols] view of a scale table: every scale over its block."""
    s = scales.repeat_interleave(g, 0)[:rows] if g > 1 else scales
    return s.repeat_interleave(128, 1)[:, :cols]


def _blocks(x, g, fill):
    """x as [rows / g][cols / 128][g * 128], the missing values filled."""
    rows, cols = x.shape
    p = torch.full((-(-rows // g) * g, -(-cols // 128) * 128), fill, device=x.device, dtype=x.dtype)
    p[:rows, :cols] = x
    return p.reshape(p.shape[0] // g, g, p.shape[1] // 128, 128).transpose(1, 2).reshape(p.shape[0] // g, -1, g * 128)


def _quantize(x, g=1):
    """Codes (float8) and exponent bytes of a matrix in 32 bits."""
    a = _blocks(torch.where(torch.isfinite(x), x.abs(), 0.0), g, 0.0).amax(2)
    m, e = torch.frexp(a)                                 # a = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(a > 0, e - 9 + (m > 0.875), 0).clamp_min(-126)
    inv = torch.ldexp(torch.ones_like(a), -e)
    scaled = torch.where(torch.isfinite(x), x, math.nan) * _spread(inv, x.shape[0], x.shape[1], g)
    return scaled.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _scale_values(b):
    """Scales as 32-bit numbers, of exponent bytes or of themselves."""
    return torch.ldexp(torch.ones(b.shape, device=b.device), b.int() - 127) if b.dtype == torch.uint8 else b


def _values(codes, scales, g=1):
    return codes.float() * _spread(_scale_values(scales), codes.shape[0], codes.shape[1], g)


def _activations(T, F, g):
    """Heavy tails and 1 % of outlier channels, as in the hidden states of a language model."""
    z = torch.randn(T, F, generator=g, device=DEVICE)
    u = torch.rand(2, T, F, generator=g, device=DEVICE).clamp_min(1e-7)
    x = z * torch.rsqrt(-(torch.log(u[0]) + torch.log(u[1])) * 0.5)          # Student t, 4 degrees of freedom
    x[:, torch.randperm(F, generator=g, device=DEVICE)[:max(1, round(0.01 * F))]] *= 20.0
    return x


def _gradients(T, n, g):
    """Small numbers, their size a token's own."""
    size = 1e-3 * torch.exp(torch.randn(T, 1, generator=g, device=DEVICE))
    return torch.randn(T, n, generator=g, device=DEVICE) * size


def _weights(case, g):
    """Codes, scales and rows per scale of the layer's weights [O][F]."""
    O, F = case["O"], case["F"]
    W = torch.randn(O, F, generator=g, device=DEVICE) * 0.02
    if case["weights"] == "solved":                       # round to nearest; the library starts there
        s = W.abs().amax(1, keepdim=True) / 7.0
        q = torch.round(W / s).clamp(-8, 7)
        return q.to(torch.float8_e4m3fn), s.expand(O, -(-F // 128)), 1
    if case["weights"] == "f32":
        s = _blocks(W, 128, 0.0).abs().amax(2) / 448.0
        q = (W / _spread(s, O, F, 128)).clamp(-448.0, 448.0)
        return q.to(torch.float8_e4m3fn), s, 128
    return *_quantize(W, 128), 128


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    op, T, F, dt = case["op"], case["T"], case["F"], TYPES[case["dtype"]]
    d = {}
    if op in ("norm", "norm_grad", "save"):
        d["x"] = _activations(T, F, g).to(dt)
    if op in ("norm", "norm_grad"):
        d["gamma"] = 1.0 + 0.1 * torch.randn(F, generator=g, device=DEVICE)
        d["beta"] = 0.1 * torch.randn(F, generator=g, device=DEVICE)
    if op == "norm_grad":
        x = d["x"].float()
        mean = x.mean(1)
        d["mean"], d["rstd"] = mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)
        d["dy"] = _gradients(T, F, g).to(dt)
        if case["from_8bit"]:
            d["x"] = (*_quantize(x), 1)
    if op in ("product", "backward"):
        a = _activations(T, F, g)
        if case["weights"] == "f32":
            s = _blocks(a, 1, 0.0).abs().amax(2) / 448.0
            d["x"] = ((a / _spread(s, T, F, 1)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), s, 1)
        else:
            d["x"] = (*_quantize(a), 1)
        d["w"] = _weights(case, g)
        if op == "product":
            d["bias"] = 0.1 * torch.randn(case["O"], generator=g, device=DEVICE)
        else:
            d["dy"] = _gradients(T, case["O"], g).to(dt)
    return d


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if own:
        from paper_2508_13437_amd import dmmv

        for k in ("x", "w"):                              # weights and checkpoints that a program holds
            if isinstance(state.get(k), tuple):
                state[k] = dmmv.BlockMatrix(*state[k])
    return state


# --------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2508_13437_amd import dmmv

    case = s["case"]
    op, dt = case["op"], TYPES[case["dtype"]]
    if op == "norm":
        if case["out"] == "8bit":
            r = dmmv.dmmv_layernorm(s["x"], s["gamma"], s["beta"], EPS, y=False, q=True)
            return {"y": dmmv.dmmv_block_dequantize(r.q, dt), "mean": r.mean, "rstd": r.rstd}
        r = dmmv.dmmv_layernorm(s["x"], s["gamma"], s["beta"], EPS, y=True, xq=True)
        return {"y": r.y, "x": r.xq.values8, "x_scale": r.xq.scales, "mean": r.mean, "rstd": r.rstd}
    if op == "norm_grad":
        dx, dgamma, dbeta = dmmv.dmmv_layernorm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "save":
        q = dmmv.dmmv_block_quantize(s["x"])
        r = {"x": q.values8, "x_scale": q.scales}
        return {**r, "back": dmmv.dmmv_block_dequantize(q, dt)} if case["restore"] else r
    if op == "product":
        return {"y": dmmv.dmmv_block_product(s["x"], s["w"], s["bias"], dtype=dt)}
    dx, dw, dbias = dmmv.dmmv_block_backward(s["dy"], s["x"], s["w"], dw=case["dw"], dbias=case["dw"])
    return {"dx": dx, "dw": dw, "dbias": dbias} if case["dw"] else {"dx": dx}


def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], TYPES[case["dtype"]]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = torch.rsqrt(c.square().mean(1) + EPS)
        y = c * rstd[:, None] * s["gamma"] + s["beta"]
        if case["out"] == "8bit":
            return {"y": _values(*_quantize(y)).to(dt), "mean": mean, "rstd": rstd}
        q, b = _quantize(x)
        return {"y": y.to(dt), "x": q, "x_scale": b, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        x = _values(*s["x"]) if case["from_8bit"] else s["x"].float()
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        h = (x - s["mean"][:, None]) * rstd
        a = dy * s["gamma"]
        dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        return {"dx": dx.to(dt), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}
    if op == "save":
        q, b = _quantize(s["x"].float())
        r = {"x": q, "x_scale": b}
        return {**r, "back": _values(q, b).to(dt)} if case["restore"] else r
    x, w = _values(*s["x"]), _values(*s["w"])
    if op == "product":
        return {"y": (x @ w.t() + s["bias"]).to(dt)}
    dy = s["dy"].float()
    dx = (dy @ w).to(dt)
    return {"dx": dx, "dw": dy.t() @ x, "dbias": dy.sum(0)} if case["dw"] else {"dx": dx}


# --------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------
def work(case):
    op, T, F, w = case["op"], case["T"], case["F"], WIDTH[case["dtype"]]
    n = float(T) * F
    eight = n * (1.0 + 1.0 / 128.0)                       # an activation in 8 bits and its scales
    if op == "norm":
        out = n * w if case["out"] == "8bit" else n * w + eight
        return {"bytes": n * w + out + 8.0 * (T + F), "flops": 10.0 * n}
    if op == "norm_grad":
        return {"bytes": 2.0 * n * w + (eight if case["from_8bit"] else n * w) + 8.0 * T + 12.0 * F, "flops": 15.0 * n}
    if op == "save":
        return {"bytes": n * w + eight + (n * w if case["restore"] else 0.0), "flops": 3.0 * n}
    O = case["O"]
    layer = float(O) * F
    if op == "product":
        return {"bytes": eight + layer + 4.0 * O + float(T) * O * w, "flops": 2.0 * n * O}
    parts = 2 if case["dw"] else 1
    return {"bytes": float(T) * O * w + layer + n * w + (eight + 4.0 * layer + 4.0 * O if case["dw"] else 0.0),
            "flops": 2.0 * n * O * parts}


# --------------------------------------------------------------------------------------
# the same numbers in 64 bits
# --------------------------------------------------------------------------------------
def _exact_blocks(x):
    """Values on the e4m3 grid and exponents, one scale per row and 128 columns, of finite x."""
    T, F = x.shape
    nb = -(-F // 128)
    pad = torch.nn.functional.pad(x, (0, nb * 128 - F)).view(T, nb, 128)
    a = pad.abs().amax(2)
    need = a / 448.0
    e = torch.ceil(torch.log2(torch.where(a > 0, need, 1.0)))
    e = torch.where(need > torch.exp2(e), e + 1, torch.where(need <= torch.exp2(e - 1), e - 1, e))
    e = torch.where(a > 0, e.clamp(min=-126), 0.0)
    v = pad / torch.exp2(e)[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).view(T, -1)[:, :F], e


def _exact_values(q, scales, rows_per_scale):
    rows, cols = q.shape
    s = torch.exp2(scales.double() - 127.0) if scales.dtype == torch.uint8 else scales.double()
    i = torch.div(torch.arange(rows, device=q.device), rows_per_scale, rounding_mode="floor")
    j = torch.div(torch.arange(cols, device=q.device), 128, rounding_mode="floor")
    return q.double() * s[i][:, j]


def exact(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        g = d["gamma"].double()
        x = _exact_values(*d["x"]) if isinstance(d["x"], tuple) else d["x"].double()
    if op == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * g + d["beta"].double()
        if case["out"] == "8bit":
            v, e = _exact_blocks(y)
            y = v * torch.exp2(e).repeat_interleave(128, 1)[:, :case["F"]]
            return {"y": y, "mean": mean, "rstd": rstd}
        return {"y": y, "x": _exact_blocks(x)[0], "x_scale": None, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        dy, n = d["dy"].double(), float(case["F"])
        r = d["rstd"].double()[:, None]
        h = (x - d["mean"].double()[:, None]) * r
        p = g[None, :] * dy
        dx = r / n * (n * p - p.sum(1)[:, None] - h * (p * h).sum(1)[:, None])
        return {"dx": dx, "dgamma": torch.einsum("tf,tf->f", dy, h), "dbeta": torch.einsum("tf->f", dy)}
    if op == "save":
        v, e = _exact_blocks(d["x"].double())
        back = v * torch.exp2(e).repeat_interleave(128, 1)[:, :case["F"]]
        return {"x": v, "x_scale": None, **({"back": back} if case["restore"] else {})}
    w = _exact_values(*d["w"])
    if op == "product":
        return {"y": torch.addmm(d["bias"].double(), _exact_values(*d["x"]), w.t())}
    dy = d["dy"].double()
    if not case["dw"]:
        return {"dx": dy @ w}
    return {"dx": dy @ w, "dw": (_exact_values(*d["x"]).t() @ dy).t(), "dbias": dy.sum(0)}
