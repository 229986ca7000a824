"""The operators of a residual block (include/dmmv_layer.h) in 64 bits, from their definitions (CPU, numpy)."""
import math

import numpy as np
from scipy.special import erfc, expit

ACTS = ("relu", "gelu", "gelu_tanh", "silu")
K = math.sqrt(2.0 / math.pi)


def act(u, kind):
    if kind is None:
        return u
    if kind == "relu":
        return np.maximum(u, 0.0)
    if kind == "gelu":
        return u * 0.5 * erfc(-u / math.sqrt(2.0))
    return u * expit(u if kind == "silu" else 2.0 * K * (u + 0.044715 * u ** 3))


def slope(u, kind):
    if kind == "relu":
        return (u > 0).astype(np.float64)
    if kind == "gelu":
        return 0.5 * erfc(-u / math.sqrt(2.0)) + u * np.exp(-u * u / 2.0) / math.sqrt(2.0 * math.pi)
    x, grow = (u, 1.0) if kind == "silu" else (2.0 * K * (u + 0.044715 * u ** 3), 2.0 * K * (1.0 + 3 * 0.044715 * u ** 2))
    return expit(x) + u * expit(x) * expit(-x) * grow


def stats(x, eps, rms):
    mean = np.zeros(len(x)) if rms else x.mean(1)
    return mean, 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)


def spread_gate(gate, rows, gate_rows):
    return 1.0 if gate is None else gate[np.arange(rows) // (gate_rows or max(rows, 1))]


def residual(f, h, post, pre, gate, alpha):
    """post, pre: None or (gamma, beta, eps, rms); gate: 1 or spread over the rows.  v, y and the statistics."""
    out, p = {}, f
    if post:
        m, r = out["post_mean"], out["post_rstd"] = stats(f, *post[2:])
        p = (f - m[:, None]) * r[:, None] * post[0] + post[1]
    v = out["h"] = alpha * h + gate * p
    if pre:
        m, r = out["mean"], out["rstd"] = stats(v, *pre[2:])
        out["y"] = (v - m[:, None]) * r[:, None] * pre[0] + pre[1]
    return out


def norm_back(a, n, rstd, rms):
    d = a - n * (a * n).mean(1, keepdims=True)
    return rstd[:, None] * (d if rms else d - a.mean(1, keepdims=True))


def residual_back(dy, dv, f, v, post, pre, gate, alpha, s):
    """s: the statistics of the forward pass.  The sums over rows come as their terms, [rows][cols]."""
    out, e = {}, np.zeros_like(f) if dv is None else dv
    if pre:
        n = (v - s["mean"][:, None]) * s["rstd"][:, None]
        e = e + norm_back(dy * pre[0], n, s["rstd"], pre[3])
        out["dgamma"], out["dbeta"] = dy * n, dy
    d, p = gate * e, f
    out["df"] = d
    if post:
        m = (f - s["post_mean"][:, None]) * s["post_rstd"][:, None]
        out["df"] = norm_back(d * post[0], m, s["post_rstd"], post[3])
        out["dpost_gamma"], out["dpost_beta"] = d * m, d
        p = m * post[0] + post[1]
    out["dh"], out["dgate"] = alpha * e, e * p
    return out
