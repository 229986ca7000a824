"""The norms around a block with its gate and residual scale, and their gradients, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import residual_plain as rp
from tests.test_gpu_block_linear import check_q
from tests.test_gpu_block_product import f64, half_ulp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# every team size and the walks over long rows, one column, odd ends
SIZES = [(1, 1), (3, 2), (5, 7), (9, 96), (4, 511), (66, 512), (7, 513), (5, 1024), (33, 1003), (3, 2048), (2, 2049), (17, 4096), (1, 4096), (3, 4100), (2, 8192),
         (3, 8193), (2, 16384), (2, 16391), (1, 40000), (300, 130)]
# post, pre, gate ("one", or rows a gate), alpha
FORMS = [("none", "layer", None, 1.0), ("none", "rms", 3, 0.5), ("layer", "none", "one", 1.0), ("rms", "none", None, -1.25), ("layer", "layer", "one", 0.75),
         ("rms", "rms", 2, 1.0), ("layer", "rms", 1, 1.0)]


def make(rows, cols, dtype, seed, device, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + pad, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    x[:, ::97] *= 20.0
    return x.to(dtype).to(device)[:, pad:]


def setup(rows, cols, form, seed, device):
    from paper_2508_13437_amd import dmmv

    g = torch.Generator().manual_seed(seed)
    post, pre, gate, alpha = form

    def norm(kind, eps):
        if kind == "none":
            return None
        beta = (0.3 * torch.randn(cols, generator=g)).to(device) if kind == "layer" else None
        return dmmv.Norm((1.0 + 0.2 * torch.randn(cols, generator=g)).to(device), beta, eps, rms=kind == "rms")

    a, b = norm(post, 1e-5), norm(pre, 1e-6)
    if gate is None:
        return a, b, None, None, alpha
    per = None if gate == "one" else gate
    n = 1 if per is None else -(-rows // per)
    return a, b, (0.6 + 0.3 * torch.randn(n, cols, generator=g)).to(device), per, alpha


def plain_norm(n, cols):
    if n is None:
        return None
    one = np.ones(cols)
    return (f64(n.gamma) if n.gamma is not None else one), (f64(n.beta) if n.beta is not None else 0 * one), float(np.float32(n.eps)), n.rms


def terms(cols):
    """Roundings on the way of a row's sum: a lane's own terms one after the other, then a tree of at most 1024 lanes."""
    return 8 * max(1, -(-cols // 8192), min(4, -(-cols // 2048)), -(-cols // 2048) if cols > 4096 else 1) + 16 + 10


def norm_error(x, e_x, n, mean, rstd, y):
    """Errors of mean, rstd (relative) and y of a norm of x, whose numbers are off by e_x."""
    k = terms(x.shape[1])
    e_mean = 0.0 * mean if n[3] else e_x.mean(1) + (k + 2) * U * np.abs(x).mean(1)
    dev = np.abs(x - mean[:, None])
    e_dev = e_x + e_mean[:, None] + U * dev
    # deviations carry their errors; half of a relative error of the variance, three more roundings
    e_var = (2 * dev * e_dev + e_dev ** 2).mean(1) + (k + 3) * U * (dev ** 2).mean(1)
    rel = 0.51 * e_var * rstd ** 2 + 4 * U
    e_y = (e_dev * rstd[:, None] + dev * rstd[:, None] * (rel[:, None] + 3 * U)) * np.abs(n[0]) * 1.01 + 2 * U * np.abs(y)
    return e_mean, rel, e_y


def check_forward(f, h, post, pre, gate, per, alpha, r, dtype):
    fd, hd = f64(f), f64(h)
    rows, cols = fd.shape
    a, b = plain_norm(post, cols), plain_norm(pre, cols)
    gate = rp.spread_gate(None if gate is None else f64(gate), rows, per)
    w = rp.residual(fd, hd, a, b, gate, alpha)
    p, e_p = fd, 0.0 * fd
    if a:
        p = (fd - w["post_mean"][:, None]) * w["post_rstd"][:, None] * a[0] + a[1]
        e_mean, rel, e_p = norm_error(fd, e_p, a, w["post_mean"], w["post_rstd"], p)
        assert (np.abs(f64(r.post_mean) - w["post_mean"]) <= e_mean).all() and (np.abs(f64(r.post_rstd) - w["post_rstd"]) <= rel * w["post_rstd"]).all()
    v = w["h"]
    e_v = np.abs(gate) * e_p + U * (np.abs(alpha * hd) + 1.01 * np.abs(v) + np.abs(gate * p))
    if r.h is not None:
        assert (np.abs(f64(r.h) - v) <= e_v + half_ulp(dtype) * 1.01 * (np.abs(v) + e_v)).all()
    if b:
        e_mean, rel, e_y = norm_error(v, e_v, b, w["mean"], w["rstd"], w["y"])
        assert (np.abs(f64(r.mean) - w["mean"]) <= e_mean).all() and (np.abs(f64(r.rstd) - w["rstd"]) <= rel * w["rstd"]).all()
        if r.y is not None:
            assert (np.abs(f64(r.y) - w["y"]) <= e_y + half_ulp(dtype) * 1.01 * (np.abs(w["y"]) + e_y)).all()
        if r.q is not None:
            check_q(r.q, w["y"], e_y)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(gpu_device, rows, cols, dtype, form):
    from paper_2508_13437_amd import dmmv

    post, pre, gate, per, alpha = setup(rows, cols, form, rows + cols, gpu_device)
    for pad in (0, 1):
        f, h = make(rows, cols, dtype, rows, gpu_device, pad), make(rows, cols, dtype, cols, gpu_device, 3 * pad)
        r = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha, q=pre is not None)
        check_forward(f, h, post, pre, gate, per, alpha, r, dtype)
        assert (r.y is None) == (pre is None) and (r.post_mean is None) == (post is None)
        if pre is None:
            continue
        if dtype == torch.float32:
            q = dmmv.dmmv_block_quantize(r.y)
            assert torch.equal(q.codes, r.q.codes) and torch.equal(q.scales, r.q.scales)
        only = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha, y=False, q=True, stream=False)
        assert only.y is None and only.h is None and torch.equal(only.q.codes, r.q.codes) and torch.equal(only.q.scales, r.q.scales)
        assert torch.equal(only.mean, r.mean) and torch.equal(only.rstd, r.rstd)


def test_it_is_the_layer_norm_of_a_sum(gpu_device):
    """Without a gate and a norm after the block: the layer norm's own result on the stream in 32 bits."""
    from paper_2508_13437_amd import dmmv

    for rows, cols in ((7, 300), (3, 4096), (2, 20000)):
        f, h = make(rows, cols, torch.float32, 1, gpu_device), make(rows, cols, torch.float32, 2, gpu_device)
        r = dmmv.dmmv_residual_norm(f, h, None, dmmv.Norm(eps=1e-5))
        assert torch.equal(r.h, f + h)
        n = dmmv.dmmv_layernorm(r.h)
        # the same sums in another order of lanes
        assert float((n.y - r.y).abs().max()) <= 2e-5 and float((n.mean - r.mean).abs().max()) <= 1e-6


def test_rows_without_variance_and_what_is_not_finite(gpu_device):
    from paper_2508_13437_amd import dmmv

    for cols in (300, 20000):
        f, h = make(6, cols, torch.float32, 3, gpu_device), make(6, cols, torch.float32, 4, gpu_device)
        f[1], h[1] = 7.0, 0.0
        f[2], h[2] = 0.0, 0.0
        for rms in (False, True):
            n = dmmv.Norm(eps=1e-5, rms=rms)
            check_forward(f, h, n, n, None, None, 1.0, dmmv.dmmv_residual_norm(f, h, n, n), torch.float32)
            clean = dmmv.dmmv_residual_norm(f, h, n, n, q=True)
            g, k = f.clone(), h.clone()
            g[3, 4], k[4, 5] = float("nan"), float("inf")
            r = dmmv.dmmv_residual_norm(g, k, n, n, q=True)
            ok = [0, 1, 2, 5]
            assert r.y[3].isnan().all() and r.h[3].isnan().all() and r.y[4, 5].isnan() and torch.equal(r.y[ok], clean.y[ok])
            assert bool((r.q.codes[3] & 127 == 127).all()) and torch.equal(r.q.codes[ok], clean.q.codes[ok])
            zero = dmmv.Norm(eps=0.0, rms=rms)
            assert dmmv.dmmv_residual_norm(f, h, None, zero).y[2].isnan().all()          # 0 / 0


def check_backward(dy, dv, f, v, post, pre, gate, per, alpha, r, got, dtype):
    d = {k: None if t is None else f64(t) for k, t in dict(dy=dy, dv=dv, f=f, v=v).items()}
    rows, cols = d["f"].shape
    a, b = plain_norm(post, cols), plain_norm(pre, cols)
    G = rp.spread_gate(None if gate is None else f64(gate), rows, per)
    s = {k: None if t is None else f64(t) for k, t in dict(post_mean=r.post_mean, post_rstd=r.post_rstd, mean=r.mean, rstd=r.rstd).items()}
    w = rp.residual_back(d["dy"], d["dv"], d["f"], d["v"], a, b, G, alpha, s)
    k = terms(cols)
    mean = lambda t: t.mean(1, keepdims=True)  # noqa: E731

    def back_error(t, e_t, n, rstd):
        """Of a norm's gradient from t, off by e_t: two roundings of n, k of the sums, the formula's six."""
        t = np.abs(t)
        return rstd[:, None] * (e_t + mean(e_t) + n * mean(e_t * n) + ((t + mean(t)) * (k + 8) + n * mean(t * n) * (k + 12)) * U) * 1.01

    e, e_e, sums = (np.zeros((rows, cols)) if d["dv"] is None else d["dv"]), np.zeros((rows, cols)), {}
    if b:
        n = np.abs((d["v"] - s["mean"][:, None]) * s["rstd"][:, None])
        e_e = back_error(d["dy"] * b[0], 0.0 * e, n, s["rstd"])
        e = e + rp.norm_back(d["dy"] * b[0], (d["v"] - s["mean"][:, None]) * s["rstd"][:, None], s["rstd"], b[3])
        e_e = e_e + U * np.abs(e)
        sums["dgamma"], sums["dbeta"] = 3 * U * np.abs(d["dy"]) * n, 0.0 * e
    g = np.abs(G)
    D, e_d = np.abs(G * e), g * e_e + U * np.abs(G * e)
    e_f, p, e_p = e_d, np.abs(d["f"]), 0.0 * e
    if a:
        m = np.abs((d["f"] - s["post_mean"][:, None]) * s["post_rstd"][:, None])
        e_f = back_error(G * e * a[0], np.abs(a[0]) * e_d, m, s["post_rstd"])
        sums["dpost_gamma"], sums["dpost_beta"] = e_d * m + 3 * U * D * m, e_d
        p, e_p = np.abs(w["dgate"] / np.where(e == 0, 1, e)), 4 * U * (m * np.abs(a[0]) + np.abs(a[1]))
    assert (np.abs(f64(got.df) - w["df"]) <= e_f + half_ulp(dtype) * 1.01 * (np.abs(w["df"]) + e_f)).all()
    e_h = np.abs(alpha) * e_e + U * np.abs(w["dh"])
    assert (np.abs(f64(got.dh) - w["dh"]) <= e_h + half_ulp(dtype) * 1.01 * (np.abs(w["dh"]) + e_h)).all()
    # sums: at most `rows` additions one after another
    for name, e_s in sums.items():
        t = getattr(got, name)
        if t is not None:
            assert (np.abs(f64(t) - w[name].sum(0)) <= 1.01 * e_s.sum(0) + (rows + 20) * U * np.abs(w[name]).sum(0)).all(), name
    if gate is None:
        assert got.dgate is None
        return
    per = per or rows
    e_s = e_e * p + np.abs(e) * e_p + (min(rows, per) + 20) * U * np.abs(w["dgate"])
    for i in range(len(gate)):
        part = slice(i * per, (i + 1) * per)
        assert (np.abs(f64(got.dgate[i]) - w["dgate"][part].sum(0)) <= 1.01 * e_s[part].sum(0)).all(), i


def same(p, q):
    for name in ("df", "dh", "dgate", "dpost_gamma", "dpost_beta", "dgamma", "dbeta"):
        s, t = getattr(p, name), getattr(q, name)
        assert (s is None) == (t is None) and (s is None or torch.equal(s, t)), name


# few rows and gates; more gates than are split; gates longer than a workgroup's rows
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES + [(1500, 96), (2300, 40), (1100, 600), (1100, 2056)])
def test_backward(gpu_device, rows, cols, dtype, form):
    from paper_2508_13437_amd import dmmv

    post, pre, gate, per, alpha = setup(rows, cols, form, rows + cols, gpu_device)
    for pad in (0, 1):
        f, h = make(rows, cols, dtype, rows, gpu_device, pad), make(rows, cols, dtype, cols, gpu_device, 3 * pad)
        r = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha)
        dy = make(rows, cols, dtype, 5, gpu_device, pad) if pre else None
        dv = make(rows, cols, dtype, 6, gpu_device, 5 * pad) if pre is None or pad == 0 else None
        got = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha)
        check_backward(dy, dv, f, r.h, post, pre, gate, per, alpha, r, got, dtype)
        same(got, dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha))
        only = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha, parameters=False)
        assert torch.equal(only.df, got.df) and torch.equal(only.dh, got.dh) and only.dgate is None and only.dgamma is None and only.dpost_gamma is None
        only = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha, df=False, dh=False)
        assert only.df is None and only.dh is None
        only.df, only.dh = got.df, got.dh
        same(only, got)


@pytest.mark.parametrize("per", [1, 2, 7, 100, 600, 1199, 1200, 5000])
@pytest.mark.parametrize("cols", [40, 513, 1500, 4200])
def test_gates_of_every_length(gpu_device, cols, per):
    from paper_2508_13437_amd import dmmv

    rows = 1200
    post, pre, gate, per, alpha = setup(rows, cols, ("layer", "rms", per, 0.5), cols, gpu_device)
    f, h = make(rows, cols, torch.float32, 1, gpu_device), make(rows, cols, torch.float32, 2, gpu_device)
    r = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha)
    check_forward(f, h, post, pre, gate, per, alpha, r, torch.float32)
    dy, dv = make(rows, cols, torch.float32, 3, gpu_device), make(rows, cols, torch.float32, 4, gpu_device)
    got = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha)
    check_backward(dy, dv, f, r.h, post, pre, gate, per, alpha, r, got, torch.float32)


def test_without_f_where_nothing_needs_it(gpu_device):
    from paper_2508_13437_amd import dmmv

    for cols in (300, 5000):
        f, h = make(9, cols, torch.bfloat16, 1, gpu_device), make(9, cols, torch.bfloat16, 2, gpu_device)
        dy = make(9, cols, torch.bfloat16, 3, gpu_device)
        n = dmmv.Norm()
        r = dmmv.dmmv_residual_norm(f, h, None, n)
        same(dmmv.dmmv_residual_norm_backward(dy, None, None, r, None, n), dmmv.dmmv_residual_norm_backward(dy, None, f, r, None, n))
        gate = torch.rand(cols, device=gpu_device)
        a = dmmv.dmmv_residual_norm_backward(dy, None, None, r, None, n, gate, parameters=False)
        b = dmmv.dmmv_residual_norm_backward(dy, None, f, r, None, n, gate)
        assert torch.equal(a.df, b.df) and torch.equal(a.dh, b.dh) and b.dgate.shape == gate.shape


def test_gradient_against_differences(gpu_device):
    """The forward formula in 64 bits, differenced: sum(dy * y) + sum(dv * v) with one input moved."""
    from paper_2508_13437_amd import dmmv

    rows, cols = 5, 37
    for form in (("layer", "layer", 2, 0.75), ("rms", "rms", "one", 1.0), ("layer", "rms", 1, 1.0)):
        post, pre, gate, per, alpha = setup(rows, cols, form, 3, gpu_device)
        f, h, dy, dv = (make(rows, cols, torch.float32, i, gpu_device) for i in range(4))
        r = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha)
        got = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha)
        at = {"f": f64(f), "h": f64(h), "gate": f64(gate), "g0": plain_norm(post, cols)[0], "b0": plain_norm(post, cols)[1], "g1": plain_norm(pre, cols)[0],
              "b1": plain_norm(pre, cols)[1]}
        a, b, D, V = plain_norm(post, cols), plain_norm(pre, cols), f64(dy), f64(dv)

        def value(x):
            w = rp.residual(x["f"], x["h"], (x["g0"], x["b0"], *a[2:]), (x["g1"], x["b1"], *b[2:]), rp.spread_gate(x["gate"], rows, per), alpha)
            return (w["y"] * D).sum() + (w["h"] * V).sum()

        step = 1e-5                                            # error of the difference some 1e-9, of a gradient in 32 bits 2e-6 of the largest
        for name, g in (("f", got.df), ("h", got.dh), ("gate", got.dgate), ("g0", got.dpost_gamma), ("b0", got.dpost_beta), ("g1", got.dgamma), ("b1", got.dbeta)):
            if g is None:
                continue
            g = f64(g)
            for i in ((0,), (7,), (36,)) if g.ndim == 1 else ((0, 0), (len(g) - 1, 5), (len(g) // 2, 36)):
                up, down = ({k: v.copy() for k, v in at.items()} for _ in range(2))
                up[name][i] += step
                down[name][i] -= step
                want = (value(up) - value(down)) / (2 * step)
                assert abs(g[i] - want) <= 5e-6 * np.abs(g).max() + 1e-7, (form, name, i)


def test_a_row_that_is_not_finite_stays_in_its_row(gpu_device):
    from paper_2508_13437_amd import dmmv

    for cols in (300, 5000):
        post, pre, gate, per, alpha = setup(40, cols, ("layer", "layer", 10, 1.0), 1, gpu_device)
        f, h, dy, dv = (make(40, cols, torch.float32, i, gpu_device) for i in range(4))
        r = dmmv.dmmv_residual_norm(f, h, post, pre, gate, per, alpha)
        clean = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha)
        dy[13, 7] = float("nan")
        got = dmmv.dmmv_residual_norm_backward(dy, dv, f, r, post, pre, gate, per, alpha)
        ok = [i for i in range(40) if i != 13]
        assert torch.equal(got.df[ok], clean.df[ok]) and torch.equal(got.dh[ok], clean.dh[ok]) and got.df[13].isnan().all() and got.dh[13].isnan().all()
        assert got.dgate[1].isnan().all() and torch.equal(got.dgate[[0, 2, 3]], clean.dgate[[0, 2, 3]])
        one = [j for j in range(cols) if j != 7]
        assert got.dgamma[7].isnan() and torch.equal(got.dgamma[one], clean.dgamma[one]) and got.dpost_beta.isnan().all()


def test_no_rows_no_columns_another_stream_and_gaps(gpu_device):
    from paper_2508_13437_amd import dmmv

    n = dmmv.Norm(torch.ones(40, device=gpu_device), torch.zeros(40, device=gpu_device))
    gate = torch.ones(1, 40, device=gpu_device)
    e = torch.empty(0, 40, device=gpu_device)
    r = dmmv.dmmv_residual_norm(e, e, n, n, gate, q=True)
    g = dmmv.dmmv_residual_norm_backward(e, e, e, r, n, n, gate)
    assert g.df.shape == (0, 40) and all((t == 0).all() for t in (g.dgate, g.dpost_gamma, g.dpost_beta, g.dgamma, g.dbeta))
    e = torch.empty(300, 0, device=gpu_device)
    n = dmmv.Norm()
    r = dmmv.dmmv_residual_norm(e, e, n, n, q=True)
    assert r.y.shape == (300, 0) and r.mean.isnan().all() and r.post_rstd.isnan().all()
    assert dmmv.dmmv_residual_norm_backward(e, e, e, r, n, n).df.shape == (300, 0)
    # another stream; vectors with gaps, whose copies outlive the allocation of the results
    k = 640
    f, h = make(50, k, torch.bfloat16, 1, gpu_device), make(50, k, torch.bfloat16, 2, gpu_device)
    v = [torch.rand(k, device=gpu_device) for _ in range(5)]
    apart = [torch.stack([x, torch.zeros_like(x)], 1)[:, 0] for x in v]
    run = lambda w: dmmv.dmmv_residual_norm(f, h, dmmv.Norm(w[0], w[1]), dmmv.Norm(w[2], w[3]), w[4])  # noqa: E731
    back = lambda w, r: dmmv.dmmv_residual_norm_backward(f, h, f, r, dmmv.Norm(w[0], w[1]), dmmv.Norm(w[2], w[3]), w[4])  # noqa: E731
    want = run(v)
    grads = back(v, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for w in (v, apart):
            got = run(w)
            assert torch.equal(got.y, want.y) and torch.equal(got.h, want.h)
            same(back(w, got), grads)
    side.synchronize()


def test_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    x, n = torch.randn(4, 200, device=gpu_device), dmmv.Norm(torch.ones(200, device=gpu_device))
    gate = torch.ones(2, 200, device=gpu_device)
    for args, kw, status in (((x.half(), x.half()), {}, -3), ((x, x.bfloat16()), {}, -3), ((x, x[:3]), {}, -2), ((x, x.cpu()), {}, -6), ((x[0], x[0]), {}, -2),
                             ((x, x, dmmv.Norm(torch.ones(199, device=gpu_device))), {}, -2), ((x, x, None, dmmv.Norm(eps=-1.0)), {}, -4),
                             ((x, x, dmmv.Norm(eps=float("nan"))), {}, -4), ((x, x), dict(q=True), -1), ((x, x, n, n, gate), {}, -2),
                             ((x, x, n, n, gate, 1), {}, -2), ((x, x, n, n, gate, 0), {}, -2), ((x, x, n, n, gate.double(), 2), {}, -3),
                             ((x, x, n, n, None, None, float("inf")), {}, -4), ((x, x, n, n, gate[:, :9], 2), {}, -2)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_residual_norm(*args, **kw)
        assert e.value.status == status, (args, kw)
    r = dmmv.dmmv_residual_norm(x, x, n, n, gate, 2)
    bare = dmmv.ResidualNormResult(None, None, None, r.post_mean, r.post_rstd, r.mean, r.rstd)
    none = dmmv.ResidualNormResult(r.h, None, None, r.post_mean, None, r.mean, r.rstd)
    for args, status in (((None, x, x, r, n, n), -1), ((x, x, x, r, n, None), -1), ((None, None, x, r, n), -1), ((x, x, None, r, n, n), -1),
                         ((x, x, x, bare, n, n), -1), ((x, x, x, none, n, n), -1), ((x, x[:3], x, r, n, n), -2), ((x, x.bfloat16(), x, r, n, n), -3),
                         ((x[:3], None, x[:3], r, n, n), -2), ((x, x, x, r, n, n, gate), -2)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_residual_norm_backward(*args)
        assert e.value.status == status, args
