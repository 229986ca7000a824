"""A residual block around quantised layers, trained and served: its operators as timed cases.

    linear      u = x w^T + bias of two 8-bit matrices, v = act(u) + residual; v in the given type or in 8 bits, u if it is kept
    act_grad    du = dy act'(u) and the gradient of the bias
    resnorm     v = alpha h + gate * post(f) and pre(v): the norm after a block, its gate and residual scale, the next block's norm
    resnorm_grad  gradients of f, h, the gate and both norms' parameters
    clip        the norm over all gradients of some blocks, and the gradients scaled to it

An 8-bit matrix holds e4m3 codes [rows][cols] and scales [rows / g][cols / 128], g = 1 or 128 (both divisions rounded up); it
stands for code * scale.  Quantising takes the smallest power of two that is at least (largest |x| of the block) / 448, not
below 2^-126, and 1 for a block of zeros.  8-bit results are returned as the values that they stand for, in bf16 (exact).

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
ACTS = ("relu", "gelu", "gelu_tanh", "silu")
CLIP_EPS = 1e-6


# --------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------
# T, F, O   tokens, features, outputs (linear: F is the contraction)
# act       of linear and act_grad;  residual: something is added after it;  keep: u is an output
# out       "y" = in the case's type, "8bit" = the next product's operand
# weights   "blocks" = e4m3 with a power of two per 128 x 128 block; "solved" = the library's answer,
#           integers of 4 bits and a scale per row; "f32" = any 32-bit scales on both sides
# post, pre "none", "layer" or "rms";  gate "none", "channel" (one for all rows) or "sequence" (one for every `rows` rows)
# stream    resnorm_grad: a gradient arrives along the residual stream
# blocks    clip: gradients of that many blocks of two layers F -> O -> F with biases and norms; small: biases and norms in bf16 too
def listed():
    return [
        # serving a single token: the up-projection of an MLP with its activation, in 8 bits for the down-projection
        dict(name="linear_token", op="linear", dtype="bf16", T=1, F=4096, O=11008, act="silu", residual=False, keep=False, out="8bit", weights="blocks"),
        # a few requests at once: the down-projection of a solved layer, added to the hidden states
        dict(name="linear_requests", op="linear", dtype="bf16", T=24, F=11008, O=4096, act="none", residual=True, keep=False, out="y", weights="solved"),
        # a short batch of odd sizes with 32-bit scales, trained in 32 bits
        dict(name="linear_ragged", op="linear", dtype="f32", T=500, F=2731, O=1777, act="gelu", residual=True, keep=True, out="y", weights="f32"),
        # training: the up-projection over a whole batch, u kept for the backward pass
        dict(name="linear_up", op="linear", dtype="bf16", T=4096, F=4096, O=11008, act="gelu", residual=False, keep=True, out="y", weights="blocks"),
        # and the down-projection, added to the hidden states
        dict(name="linear_down", op="linear", dtype="bf16", T=4096, F=11008, O=4096, act="none", residual=True, keep=False, out="y", weights="blocks"),
        # backward through the activation of that batch, with the gradient of the up-projection's bias
        dict(name="act_grad", op="act_grad", dtype="bf16", T=4096, O=11008, act="gelu", dbias=True),
        # serving a single token: a block's output added to the hidden state, and the next block's norm in 8 bits
        dict(name="resnorm_token", op="resnorm", dtype="bf16", T=1, F=4096, post="none", pre="layer", gate="none", rows=0, alpha=1.0, out="8bit"),
        # training: norms on both sides of the block, a gate per channel
        dict(name="resnorm", op="resnorm", dtype="bf16", T=4096, F=4096, post="rms", pre="rms", gate="channel", rows=0, alpha=1.0, out="y"),
        # gradients, odd sizes, 32 bits, sequences of 100 tokens with gates of their own, a residual scale
        dict(name="resnorm_grad_ragged", op="resnorm_grad", dtype="f32", T=513, F=1003, post="layer", pre="layer", gate="sequence", rows=100, alpha=0.75, stream=True),
        # gradients of the training batch
        dict(name="resnorm_grad", op="resnorm_grad", dtype="bf16", T=4096, F=4096, post="rms", pre="rms", gate="channel", rows=0, alpha=1.0, stream=True),
        # a small model's gradients, odd sizes, vectors in bf16 among them
        dict(name="clip_small", op="clip", blocks=2, F=333, O=1003, small=True, clipped=True),
        # four MLP-shaped blocks in 32 bits
        dict(name="clip_layers", op="clip", blocks=4, F=4096, O=11008, small=False, clipped=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    n = _log_uniform(rng, lo, hi)
    return -(-n // 128) * 128 if rng.random() < 0.4 else n             # layers are mostly multiples of a block


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "act_grad", "resnorm", "resnorm", "resnorm_grad", "resnorm_grad", "clip", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    T = _log_uniform(rng, 1, 4096)
    if op == "linear":
        up = rng.random() < 0.5
        F, O = _size(rng, 64, 4096 if up else 11008), _size(rng, 64, 11008 if up else 4096)
        act = rng.choice(["none", *ACTS])
        # (bf16 sums over many tokens may be those of 8-bit matrix cores, which move some numbers across a border of the 8-bit grid)
        eight = (T <= 64 or dtype == "f32") and rng.random() < 0.5
        return dict(op=op, dtype=dtype, T=T, F=F, O=O, act=act, residual=act == "none" or rng.random() < 0.3,
                    keep=act != "none" and rng.random() < 0.5, out="8bit" if eight else "y", weights=rng.choice(["blocks", "solved", "f32"]))
    if op == "act_grad":
        return dict(op=op, dtype=dtype, T=T, O=_size(rng, 64, 11008), act=rng.choice(ACTS), dbias=rng.random() < 0.7)
    if op == "clip":
        return dict(op=op, blocks=rng.randint(1, 4), F=_size(rng, 16, 4096), O=_size(rng, 16, 8192), small=rng.random() < 0.5,
                    clipped=rng.random() < 0.7)
    F = _size(rng, 64, 4096)
    post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("layer", "none"), ("rms", "none"), ("layer", "layer"), ("rms", "rms"), ("layer", "rms")])
    gate = rng.choice(["none", "channel", "sequence"])
    d = dict(op=op, dtype=dtype, T=T, F=F, post=post, pre=pre, gate=gate, rows=_log_uniform(rng, 1, 1024) if gate == "sequence" else 0,
             alpha=rng.choice([1.0, 1.0, 0.75]))
    if op == "resnorm":
        return dict(d, out=rng.choice(["y", "8bit"]))
    return dict(d, stream=pre == "none" or rng.random() < 0.7)


# --------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------
def _spread(scales, rows, cols, g):
    """[rows][cols] view of a scale table: every scale over its block."""
    s = scales.repeat_interleave(g, 0)[:rows] if g > 1 else scales
    return s.repeat_interleave(128, 1)[:, :cols]


def _blocks(x, g):
    """x as [rows / g][cols / 128][g * 128], the missing values zero."""
    rows, cols = x.shape
    p = torch.zeros(-(-rows // g) * g, -(-cols // 128) * 128, device=x.device, dtype=x.dtype)
    p[:rows, :cols] = x
    return p.reshape(p.shape[0] // g, g, p.shape[1] // 128, 128).transpose(1, 2).reshape(p.shape[0] // g, -1, g * 128)


def _quantize(x, g=1):
    """Codes (float8) and exponent bytes of a finite matrix in 32 bits."""
    a = _blocks(x.abs(), g).amax(2)
    m, e = torch.frexp(a)                                 # a = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(a > 0, e - 9 + (m > 0.875), 0).clamp_min(-126)
    scaled = x * _spread(torch.ldexp(torch.ones_like(a), -e), x.shape[0], x.shape[1], g)
    return scaled.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, scales, g=1):
    s = torch.ldexp(torch.ones(scales.shape, device=scales.device), scales.int() - 127) if scales.dtype == torch.uint8 else scales
    return codes.float() * _spread(s, codes.shape[0], codes.shape[1], g)


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
    """Codes, scales and rows per scale of the layer's weights [O][F]; pre-activations come out near 1."""
    O, F = case["O"], case["F"]
    W = torch.randn(O, F, generator=g, device=DEVICE) * (0.5 / math.sqrt(F))
    if case["weights"] == "solved":                       # round to nearest; the library starts there
        s = W.abs().amax(1, keepdim=True) / 7.0
        q = torch.round(W / s).clamp(-8, 7)
        return q.to(torch.float8_e4m3fn), s.expand(O, -(-F // 128)), 1
    if case["weights"] == "f32":
        s = _blocks(W, 128).abs().amax(2) / 448.0
        q = (W / _spread(s, O, F, 128)).clamp(-448.0, 448.0)
        return q.to(torch.float8_e4m3fn), s, 128
    return *_quantize(W, 128), 128


def _vector(n, mean, size, g):
    return mean + size * torch.randn(n, generator=g, device=DEVICE)


def _norm_stats(x, kind):
    mean = x.mean(1) if kind == "layer" else torch.zeros(x.shape[0], device=x.device)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    op = case["op"]
    if op == "clip":
        F, O, N = case["F"], case["O"], case["blocks"]
        shapes = [s for _ in range(N) for s in ((O, F), (O,), (F, O), (F,), (F,), (F,))]
        size = torch.exp(torch.randn(len(shapes), generator=g, device=DEVICE)).tolist()
        grads = [torch.randn(s, generator=g, device=DEVICE).mul_(1e-3 * a) for s, a in zip(shapes, size)]
        if case["small"]:
            grads = [t.bfloat16() if t.dim() == 1 else t for t in grads]
        return {"grads": grads, "max_norm": 1e-2 if case["clipped"] else 1e6}
    T, dt = case["T"], TYPES[case["dtype"]]
    if op == "linear":
        F, O, d = case["F"], case["O"], {}
        a = _activations(T, F, g)
        if case["weights"] == "f32":
            s = _blocks(a, 1).abs().amax(2) / 448.0
            d["x"] = ((a / _spread(s, T, F, 1)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), s, 1)
        else:
            d["x"] = (*_quantize(a), 1)
        d["w"] = _weights(case, g)
        d["bias"] = _vector(O, 0.0, 0.1, g)
        d["residual"] = _activations(T, O, g).to(dt) if case["residual"] else None
        return d
    if op == "act_grad":
        return {"dy": _gradients(T, case["O"], g).to(dt), "u": (1.5 * torch.randn(T, case["O"], generator=g, device=DEVICE)).to(dt)}
    F = case["F"]
    d = {"f": _activations(T, F, g).to(dt), "h": _activations(T, F, g).to(dt), "gate": None}
    if case["gate"] != "none":
        groups = 1 if case["gate"] == "channel" else -(-T // case["rows"])
        d["gate"] = 0.5 + 0.2 * torch.randn(groups, F, generator=g, device=DEVICE)
    for k in ("post", "pre"):
        d[k + "_gamma"] = _vector(F, 1.0, 0.1, g) if case[k] != "none" else None
        d[k + "_beta"] = _vector(F, 0.0, 0.1, g) if case[k] == "layer" else None
    if op == "resnorm":
        return d
    # what the forward pass kept: the block's output, the new hidden states, the norms' statistics
    p, gate = d["f"].float(), _gate(case, d["gate"], T)
    if case["post"] != "none":
        d["post_mean"], d["post_rstd"] = _norm_stats(p, case["post"])
        p = (p - d["post_mean"][:, None]) * d["post_rstd"][:, None] * d["post_gamma"]
        p = p + d["post_beta"] if d["post_beta"] is not None else p
    v = case["alpha"] * d.pop("h").float() + gate * p
    if case["pre"] != "none":
        d["mean"], d["rstd"] = _norm_stats(v, case["pre"])
        d["dy"] = _gradients(T, F, g).to(dt)
    d["h"] = v.to(dt)
    d["dh"] = _gradients(T, F, g).to(dt) if case["stream"] else None
    return d


def _gate(case, gate, T):
    """The gate of every row, 1 without one."""
    if gate is None:
        return 1.0
    return gate if case["gate"] == "channel" else gate.repeat_interleave(case["rows"], 0)[:T]


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["op"] == "clip":                              # the raw gradients are summed on: the clipped ones have buffers of their own
        state["out"] = [torch.empty_like(t) for t in state["grads"]]
    if own:
        from paper_2508_13437_amd import dmmv

        for k in ("x", "w"):                              # 8-bit matrices that a program holds
            if isinstance(state.get(k), tuple):
                state[k] = dmmv.BlockMatrix(*state[k])
        if case["op"] == "clip":                          # a training program's gradients stay where they are
            state["grads"], state["clipped"] = dmmv.Gradients(state["grads"]), dmmv.Gradients(state["out"])
        for k in ("post", "pre"):
            if case.get(k, "none") != "none":
                state[k] = dmmv.Norm(state[k + "_gamma"], state[k + "_beta"], EPS, rms=case[k] == "rms")
    return state


# --------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2508_13437_amd import dmmv

    case = s["case"]
    op = case["op"]
    if op == "clip":
        norm = dmmv.dmmv_gradient_clip(s["grads"], s["max_norm"], CLIP_EPS, out=s["clipped"])
        return {"norm": norm, "grads": s["out"]}
    dt = TYPES[case["dtype"]]
    if op == "linear":
        r = dmmv.dmmv_block_linear(s["x"], s["w"], s["bias"], None if case["act"] == "none" else case["act"], s["residual"], dt,
                                   y=case["out"] == "y", q=case["out"] == "8bit", u=case["keep"])
        y = r.y if case["out"] == "y" else dmmv.dmmv_block_dequantize(r.q, torch.bfloat16)
        return {"y": y, "u": r.u} if case["keep"] else {"y": y}
    if op == "act_grad":
        du, dbias = dmmv.dmmv_activation_backward(s["dy"], s["u"], case["act"], dbias=case["dbias"])
        return {"du": du, "dbias": dbias} if case["dbias"] else {"du": du}
    post, pre = s.get("post"), s.get("pre")
    rows = case["rows"] or None
    if op == "resnorm":
        normed = pre is not None
        r = dmmv.dmmv_residual_norm(s["f"], s["h"], post, pre, s["gate"], rows, case["alpha"], y=normed and case["out"] == "y",
                                    q=normed and case["out"] == "8bit")
        out = {"h": r.h}
        if post is not None:
            out["post_mean"], out["post_rstd"] = r.post_mean, r.post_rstd
        if normed:
            out["mean"], out["rstd"] = r.mean, r.rstd
            out["y"] = r.y if case["out"] == "y" else dmmv.dmmv_block_dequantize(r.q, torch.bfloat16)
        return out
    kept = dmmv.ResidualNormResult(s["h"], None, None, s.get("post_mean"), s.get("post_rstd"), s.get("mean"), s.get("rstd"))
    g = dmmv.dmmv_residual_norm_backward(s.get("dy"), s["dh"], s["f"], kept, post, pre, s["gate"], rows, case["alpha"])
    out = {"df": g.df, "dh": g.dh, "dgate": g.dgate, "dpost_gamma": g.dpost_gamma, "dpost_beta": g.dpost_beta, "dgamma": g.dgamma, "dbeta": g.dbeta}
    return {k: v for k, v in out.items() if v is not None}


def _act(u, act):
    if act == "none":
        return u
    if act == "relu":
        return torch.where(u > 0, u, 0.0)
    if act == "gelu":
        return 0.5 * u * torch.special.erfc(u * -math.sqrt(0.5))
    if act == "gelu_tanh":
        u2 = math.sqrt(8.0 / math.pi) * (u + 0.044715 * u * u * u)
        return u / (1.0 + torch.exp(-u2))
    return u / (1.0 + torch.exp(-u))


def _act_slope(u, act):
    if act == "relu":
        return (u > 0).float()
    if act == "gelu":
        return 0.5 * torch.special.erfc(u * -math.sqrt(0.5)) + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(8.0 / math.pi)
        s = 1.0 / (1.0 + torch.exp(-c * (u + 0.044715 * u * u * u)))
        return s + u * s * (1.0 - s) * c * (1.0 + 3.0 * 0.044715 * u * u)
    s = 1.0 / (1.0 + torch.exp(-u))
    return s * (1.0 + u * (1.0 - s))


def _normed(x, kind, gamma, beta, mean, rstd):
    y = (x - mean[:, None] if kind == "layer" else x) * rstd[:, None] * gamma
    return y if beta is None else y + beta


def _norm_back(a, x, mean, rstd, kind):
    """The gradient of x from that of its normalised values, and those."""
    h = (x - mean[:, None]) * rstd[:, None]
    d = a - h * (a * h).mean(1, keepdim=True)
    if kind == "layer":
        d = d - a.mean(1, keepdim=True)
    return rstd[:, None] * d, h


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "clip":
        norm = torch.sqrt(torch.stack([t.double().square().sum() for t in s["grads"]]).sum())
        c = (s["max_norm"] / (norm + CLIP_EPS)).clamp_max(1.0).float()
        return {"norm": norm.float(), "grads": [o.copy_(t.float() * c) for t, o in zip(s["grads"], s["out"])]}
    dt = TYPES[case["dtype"]]
    if op == "linear":
        u = _values(*s["x"]) @ _values(*s["w"]).t() + s["bias"]
        v = _act(u, case["act"])
        if s["residual"] is not None:
            v = v + s["residual"].float()
        y = v.to(dt) if case["out"] == "y" else _values(*_quantize(v)).bfloat16()
        return {"y": y, "u": u.to(dt)} if case["keep"] else {"y": y}
    if op == "act_grad":
        du = s["dy"].float() * _act_slope(s["u"].float(), case["act"])
        return {"du": du.to(dt), "dbias": du.sum(0)} if case["dbias"] else {"du": du.to(dt)}
    T = s["f"].shape[0]
    f, gate = s["f"].float(), _gate(case, s["gate"], T)
    if op == "resnorm":
        out, p = {}, f
        if case["post"] != "none":
            out["post_mean"], out["post_rstd"] = _norm_stats(f, case["post"])
            p = _normed(f, case["post"], s["post_gamma"], s["post_beta"], out["post_mean"], out["post_rstd"])
        v = case["alpha"] * s["h"].float() + gate * p
        if case["pre"] != "none":
            out["mean"], out["rstd"] = _norm_stats(v, case["pre"])
            y = _normed(v, case["pre"], s["pre_gamma"], s["pre_beta"], out["mean"], out["rstd"])
            out["y"] = y.to(dt) if case["out"] == "y" else _values(*_quantize(y)).bfloat16()
        return {"h": v.to(dt), **out}
    out, e = {}, 0.0
    if s["dh"] is not None:
        e = s["dh"].float()
    if case["pre"] != "none":
        dy = s["dy"].float()
        back, hh = _norm_back(dy * s["pre_gamma"], s["h"].float(), s["mean"], s["rstd"], case["pre"])
        e = e + back
        out["dgamma"] = (dy * hh).sum(0)
        if s["pre_beta"] is not None:
            out["dbeta"] = dy.sum(0)
    dp = gate * e
    if case["post"] != "none":
        df, ff = _norm_back(dp * s["post_gamma"], f, s["post_mean"], s["post_rstd"], case["post"])
        p = ff * s["post_gamma"] if s["post_beta"] is None else ff * s["post_gamma"] + s["post_beta"]
        out["dpost_gamma"] = (dp * ff).sum(0)
        if s["post_beta"] is not None:
            out["dpost_beta"] = dp.sum(0)
    else:
        df, p = dp, f
    if case["gate"] != "none":
        n, rows = s["gate"].shape[0], case["rows"] or T
        ep = torch.zeros(n * rows, f.shape[1], device=f.device)
        ep[:T] = e * p
        out["dgate"] = ep.view(n, rows, -1).sum(1)
    return {"df": df.to(dt), "dh": (case["alpha"] * e).to(dt), **out}


# --------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------
def work(case):
    op, F = case["op"], float(case.get("F", 0))
    if op == "clip":
        O, N = float(case["O"]), case["blocks"]
        big, small = 2.0 * O * F * N, (O + 3.0 * F) * N
        return {"bytes": 2.0 * (4.0 * big + (2.0 if case["small"] else 4.0) * small), "flops": 3.0 * (big + small)}
    T, w = float(case["T"]), WIDTH[case["dtype"]]
    if op == "linear":
        O = float(case["O"])
        out = T * O * ((w if case["residual"] else 0) + (w if case["keep"] else 0) + (w if case["out"] == "y" else 2))
        return {"bytes": T * F * (1.0 + 1.0 / 128.0) + O * F + 4.0 * O + out, "flops": 2.0 * T * O * F}
    if op == "act_grad":
        n = T * case["O"]
        return {"bytes": 3.0 * n * w + (4.0 * case["O"] if case["dbias"] else 0.0), "flops": 20.0 * n}
    n = T * F
    vectors = 4.0 * F * ((case["post"] != "none") + (case["post"] == "layer") + (case["pre"] != "none") + (case["pre"] == "layer"))
    groups = {"none": 0, "channel": 1, "sequence": -(-case["T"] // case["rows"]) if case["rows"] else 0}[case["gate"]]
    stats = 8.0 * T * ((case["post"] != "none") + (case["pre"] != "none"))
    if op == "resnorm":
        out = 0.0 if case["pre"] == "none" else n * (w if case["out"] == "y" else 2)
        return {"bytes": 3.0 * n * w + out + vectors + 4.0 * F * groups + stats, "flops": 20.0 * n}
    # f is not needed where there is neither a norm after the block nor a gate, h where there is none before
    reads = (case["post"] != "none" or case["gate"] != "none") + 2.0 * (case["pre"] != "none") + (1.0 if case["stream"] else 0.0)
    return {"bytes": (reads + 2.0) * n * w + 2.0 * vectors + 8.0 * F * groups + stats, "flops": 30.0 * n}


# --------------------------------------------------------------------------------------
# the same numbers in 64 bits
# --------------------------------------------------------------------------------------
def _exact_eight(x):
    """The values that finite x [T][F] has in 8 bits, one power of two per row and 128 columns."""
    T, F = x.shape
    nb = -(-F // 128)
    pad = torch.nn.functional.pad(x, (0, nb * 128 - F)).view(T, nb, 128)
    need = pad.abs().amax(2) / 448.0
    e = torch.ceil(torch.log2(torch.where(need > 0, need, 1.0)))
    e = torch.where(need > torch.exp2(e), e + 1, torch.where(need <= torch.exp2(e - 1), e - 1, e))
    scale = torch.exp2(torch.where(need > 0, e.clamp(min=-126), 0.0))[:, :, None]
    v = pad / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step * scale).view(T, -1)[:, :F]


def _exact_values(q, scales, rows_per_scale):
    rows, cols = q.shape
    s = torch.exp2(scales.double() - 127.0) if scales.dtype == torch.uint8 else scales.double()
    i = torch.div(torch.arange(rows, device=q.device), rows_per_scale, rounding_mode="floor")
    j = torch.div(torch.arange(cols, device=q.device), 128, rounding_mode="floor")
    return q.double() * s[i][:, j]


def _exact_normal(u):
    """The normal distribution's function and density."""
    return 0.5 * torch.special.erfc(-u / math.sqrt(2.0)), torch.exp(-u * u / 2.0) / math.sqrt(2.0 * math.pi)


def _exact_act(u, act):
    k = math.sqrt(2.0 / math.pi)
    return {"none": lambda: u, "relu": lambda: u.clamp(min=0.0), "gelu": lambda: u * _exact_normal(u)[0],
            "gelu_tanh": lambda: u * torch.sigmoid(2.0 * k * (u + 0.044715 * u ** 3)), "silu": lambda: u * torch.sigmoid(u)}[act]()


def _exact_slope(u, act):
    if act == "relu":
        return torch.where(u > 0, 1.0, 0.0).double()
    if act == "gelu":
        area, density = _exact_normal(u)
        return area + u * density
    inner, grow = (u, 1.0) if act == "silu" else (2.0 * math.sqrt(2.0 / math.pi) * (u + 0.044715 * u ** 3),
                                                  2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * u ** 2))
    s, t = torch.sigmoid(inner), torch.sigmoid(-inner)
    return s + u * s * t * grow


def exact(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    if op == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t.double().flatten()) for t in d["grads"]]))
        c = min(1.0, d["max_norm"] / (float(norm) + CLIP_EPS))
        return {"norm": norm, "grads": [t.double() * c for t in d["grads"]]}
    if op == "linear":
        u = torch.addmm(d["bias"].double(), _exact_values(*d["x"]), _exact_values(*d["w"]).t())
        v = _exact_act(u, case["act"])
        if d["residual"] is not None:
            v = d["residual"].double() + v
        return {"y": v if case["out"] == "y" else _exact_eight(v), **({"u": u} if case["keep"] else {})}
    if op == "act_grad":
        du = _exact_slope(d["u"].double(), case["act"]) * d["dy"].double()
        return {"du": du, "dbias": torch.einsum("to->o", du)} if case["dbias"] else {"du": du}
    f = d["f"].double()
    T, F = f.shape
    gate = torch.ones(T, F, dtype=torch.float64, device=f.device)
    row = torch.arange(T, device=f.device)
    group = torch.div(row, case["rows"] or T, rounding_mode="floor")
    if d["gate"] is not None:
        gate = d["gate"].double()[group]
    g0, b0 = (t if t is None else t.double() for t in (d["post_gamma"], d["post_beta"]))
    g1, b1 = (t if t is None else t.double() for t in (d["pre_gamma"], d["pre_beta"]))
    out = {}
    if op == "resnorm":
        def norm(x, kind, g, b):
            m = x.sum(1) / F * (kind == "layer")
            r = 1.0 / torch.sqrt((x - m[:, None]).pow(2).sum(1) / F + EPS)
            y = g * ((x - m[:, None]) * r[:, None])
            return m, r, y if b is None else y + b
        p = f
        if case["post"] != "none":
            out["post_mean"], out["post_rstd"], p = norm(f, case["post"], g0, b0)
        v = gate * p + d["h"].double() * case["alpha"]
        out["h"] = v
        if case["pre"] != "none":
            out["mean"], out["rstd"], y = norm(v, case["pre"], g1, b1)
            out["y"] = y if case["out"] == "y" else _exact_eight(y)
        return out

    def back(a, x, mean, rstd, kind):
        n = (x - mean.double()[:, None]) * rstd.double()[:, None]
        whole = F * a - n * torch.einsum("tf,tf->t", a, n)[:, None]
        if kind == "layer":
            whole = whole - a.sum(1)[:, None]
        return whole * (rstd.double()[:, None] / F), n
    e = torch.zeros_like(f) if d["dh"] is None else d["dh"].double()
    if case["pre"] != "none":
        dy = d["dy"].double()
        through, n = back(g1 * dy, d["h"].double(), d["mean"], d["rstd"], case["pre"])
        e = e + through
        out["dgamma"] = torch.einsum("tf,tf->f", dy, n)
        if b1 is not None:
            out["dbeta"] = torch.einsum("tf->f", dy)
    p, df = f, gate * e
    if case["post"] != "none":
        out_grad = gate * e
        df, n = back(g0 * out_grad, f, d["post_mean"], d["post_rstd"], case["post"])
        p = n * g0 if b0 is None else n * g0 + b0
        out["dpost_gamma"] = torch.einsum("tf,tf->f", out_grad, n)
        if b0 is not None:
            out["dpost_beta"] = torch.einsum("tf->f", out_grad)
    if d["gate"] is not None:
        out["dgate"] = torch.zeros(d["gate"].shape, dtype=torch.float64, device=f.device).index_add_(0, group, e * p)
    return {"df": df, "dh": case["alpha"] * e, **out}
