"""Layer norm and its gradients against 64 bits."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# every team size and the walk over long rows, one column, odd ends
SIZES = [(1, 1), (3, 2), (5, 7), (9, 96), (4, 511), (66, 512), (7, 513), (5, 1024), (33, 1003), (3, 2048), (2, 2049), (17, 4096),
         (3, 4100), (2, 8192), (3, 8193), (2, 16384), (2, 16391), (1, 40000)]


def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U      # 8 and 24 significant bits


def make(rows, cols, dtype, seed, device, pad=0, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + pad, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) + offset
    x[:, ::97] *= 20.0
    return x.to(dtype).to(device)[:, pad:]


def vectors(cols, seed, device):
    g = torch.Generator().manual_seed(seed)
    return (1.0 + 0.2 * torch.randn(cols, generator=g)).to(device), (0.3 * torch.randn(cols, generator=g)).to(device)


def f64(t):
    return t.double().cpu().numpy()


def terms(cols):
    """Roundings on the way of a row's sum: a lane's own terms one after the other, then a tree of at most 1024 lanes."""
    return 8 * max(1, -(-cols // 8192), min(4, -(-cols // 2048))) + 16 + 10


def check_forward(x, gamma, beta, eps, r, dtype):
    xd = f64(x)
    cols = xd.shape[1]
    want, mean, rstd = plain.norm(xd, f64(gamma), f64(beta), eps)
    n = terms(cols)
    at = np.abs(xd).mean(1)
    e_mean = (n + 2) * U * at                                        # of the sum, of the division
    assert (np.abs(f64(r.mean) - mean) <= e_mean).all()
    # deviations carry the mean's error and their own rounding; half of a relative error of the variance, three more roundings
    dev = np.abs(xd - mean[:, None])
    e_var = (2 * dev * (e_mean[:, None] + U * dev) + e_mean[:, None] ** 2).mean(1) + (n + 3) * U * (dev ** 2).mean(1)
    rel = 0.51 * e_var * rstd ** 2 + 4 * U
    assert (np.abs(f64(r.rstd) - rstd) <= rel * rstd).all()
    h = dev * rstd[:, None]
    e_v = ((e_mean[:, None] * rstd[:, None]) + h * (rel[:, None] + 3 * U)) * np.abs(f64(gamma)) * 1.01 + 2 * U * np.abs(want)
    if r.y is not None:
        assert (np.abs(f64(r.y) - want) <= e_v + half_ulp(dtype) * 1.01 * (np.abs(want) + e_v)).all()
    return want, e_v


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(gpu_device, rows, cols, dtype):
    from paper_2508_13437_amd import dmmv

    for pad in (0, 1):
        x = make(rows, cols, dtype, 31 * rows + cols, gpu_device, pad)
        gamma, beta = vectors(cols, cols, gpu_device)
        r = dmmv.dmmv_layernorm(x, gamma, beta, 1e-5, y=True, q=True, xq=True)
        _, e_v = check_forward(x, gamma, beta, 1e-5, r, dtype)
        # the checkpoint of the input is the quantised input, bit for bit
        q = dmmv.dmmv_block_quantize(x)
        assert torch.equal(q.codes, r.xq.codes) and torch.equal(q.scales, r.xq.scales)
        # the 8-bit result is that of the 32-bit values
        if dtype == torch.float32:
            q = dmmv.dmmv_block_quantize(r.y)
            assert torch.equal(q.codes, r.q.codes) and torch.equal(q.scales, r.q.scales)
        else:
            want = plain.norm(f64(x), f64(gamma), f64(beta), 1e-5)[0]
            step = plain.spread(plain.scale_values(r.q.scales.cpu().numpy()), rows, cols, 1) * 2.0 ** -10
            got = plain.values(r.q.codes.cpu().numpy(), r.q.scales.cpu().numpy())
            assert (np.abs(got - want) <= e_v + np.maximum(2.0 ** -4 * (np.abs(want) + e_v), step)).all()
        only = dmmv.dmmv_layernorm(x, gamma, beta, 1e-5, y=False, q=True)
        assert only.y is None and only.xq is None and torch.equal(only.q.codes, r.q.codes) and torch.equal(only.q.scales, r.q.scales)


def test_rows_without_variance_large_offsets_and_no_parameters(gpu_device):
    from paper_2508_13437_amd import dmmv

    one = torch.ones(300, device=gpu_device)
    x = make(6, 300, torch.float32, 3, gpu_device, offset=3.0e4)
    x[1] = 7.0
    x[2] = 0.0
    r = dmmv.dmmv_layernorm(x, eps=1e-5)
    check_forward(x, one, 0 * one, 1e-5, r, torch.float32)
    assert (r.y[2] == 0).all() and float(r.mean[1]) == 7.0
    x[3, 4], x[4, 5] = float("nan"), float("inf")
    r = dmmv.dmmv_layernorm(x, eps=0.0)
    assert r.y[3:5].isnan().all() and r.y[0].isfinite().all()          # a row's own, and no other's
    assert r.y[2].isnan().all()                                        # eps = 0: 0 / 0


@pytest.mark.parametrize("from_8bit", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES + [(700, 96), (1500, 520)])
def test_backward(gpu_device, rows, cols, dtype, from_8bit):
    from paper_2508_13437_amd import dmmv

    for pad in (0, 1):
        x = make(rows, cols, dtype, 7 * rows + cols, gpu_device, pad)
        dy = make(rows, cols, dtype, 11 * rows + cols, gpu_device, 3 * pad)
        gamma, beta = vectors(cols, cols, gpu_device)
        r = dmmv.dmmv_layernorm(x, gamma, beta, 1e-5, y=False, xq=True)
        got = dmmv.dmmv_layernorm_backward(dy, r.xq if from_8bit else x, gamma, r.mean, r.rstd)
        xd = plain.values(r.xq.codes.cpu().numpy(), r.xq.scales.cpu().numpy()) if from_8bit else f64(x)
        mu, rs, g, d = f64(r.mean), f64(r.rstd), f64(gamma), f64(dy)
        dx, dg, db = plain.norm_grad(d, xd, g, mu, rs)
        h = np.abs((xd - mu[:, None]) * rs[:, None])
        a = np.abs(d * g)
        n = terms(cols)
        # two roundings of h, one of a, n of the sums, the rest of the formula's five
        e = rs[:, None] * ((a + a.mean(1, keepdims=True)) * (n + 8) + h * (a * h).mean(1, keepdims=True) * (n + 12)) * U
        assert (np.abs(f64(got[0]) - dx) <= e + half_ulp(dtype) * 1.01 * (np.abs(dx) + e)).all()
        # at most `rows` additions one after another, and two roundings of h
        assert (np.abs(f64(got[1]) - dg) <= (rows + 20) * U * (np.abs(d) * h).sum(0)).all()
        assert (np.abs(f64(got[2]) - db) <= (rows + 20) * U * np.abs(d).sum(0)).all()
        again = dmmv.dmmv_layernorm_backward(dy, r.xq if from_8bit else x, gamma, r.mean, r.rstd)
        assert all(torch.equal(p, q) for p, q in zip(got, again))
        parts = [dmmv.dmmv_layernorm_backward(dy, r.xq if from_8bit else x, gamma, r.mean, r.rstd, dx=i == 0, dgamma=i == 1, dbeta=i == 2)
                 for i in range(3)]
        for i in range(3):
            assert torch.equal(parts[i][i], got[i]) and all(parts[i][j] is None for j in range(3) if j != i)


def test_gradient_against_differences(gpu_device):
    """The forward formula in 64 bits, differenced: sum(dy * norm(x)) with one input moved."""
    from paper_2508_13437_amd import dmmv

    rows, cols = 3, 37
    x, dy = make(rows, cols, torch.float32, 1, gpu_device), make(rows, cols, torch.float32, 2, gpu_device)
    gamma, beta = vectors(cols, 4, gpu_device)
    r = dmmv.dmmv_layernorm(x, gamma, beta, 1e-5)
    dx, dg, db = (f64(t) for t in dmmv.dmmv_layernorm_backward(dy, x, gamma, r.mean, r.rstd))
    X, D, G, B = f64(x), f64(dy), f64(gamma), f64(beta)
    step = 1e-5                                                        # error of the difference about 1e-10, of a gradient 1e-6
    for i, j in ((0, 0), (1, 5), (2, 36)):
        p, m = X.copy(), X.copy()
        p[i, j] += step
        m[i, j] -= step
        want = ((plain.norm(p, G, B, 1e-5)[0] - plain.norm(m, G, B, 1e-5)[0]) * D).sum() / (2 * step)
        assert abs(dx[i, j] - want) <= 2e-6 * np.abs(dx).max()
    for j in (0, 17, 36):
        p, m = G.copy(), G.copy()
        p[j] += step
        m[j] -= step
        want = ((plain.norm(X, p, B, 1e-5)[0] - plain.norm(X, m, B, 1e-5)[0]) * D).sum() / (2 * step)
        assert abs(dg[j] - want) <= 2e-6 * np.abs(dg).max()
        assert abs(db[j] - D[:, j].sum()) <= 2e-6 * np.abs(db).max()


def test_vectors_with_gaps(gpu_device):
    """Copies of strided vectors outlive the allocation of the results, which have their size here."""
    from paper_2508_13437_amd import dmmv

    n = 640
    x = make(n, n, torch.float32, 12, gpu_device)
    gamma, beta = vectors(n, 13, gpu_device)
    apart = [torch.stack([v, torch.zeros_like(v)], 1)[:, 0] for v in (gamma, beta)]
    r, s = dmmv.dmmv_layernorm(x, gamma, beta, xq=True), dmmv.dmmv_layernorm(x, *apart, xq=True)
    for a, b in ((r.y, s.y), (r.mean, s.mean), (r.rstd, s.rstd), (r.xq.codes, s.xq.codes)):
        assert torch.equal(a, b)
    stats = [torch.stack([v, torch.zeros_like(v)], 1)[:, 0] for v in (r.mean, r.rstd)]
    for a, b in zip(dmmv.dmmv_layernorm_backward(x, x, gamma, r.mean, r.rstd), dmmv.dmmv_layernorm_backward(x, x, apart[0], *stats)):
        assert torch.equal(a, b)
    row = dmmv.dmmv_block_quantize(x[:1])
    assert torch.equal(dmmv.dmmv_block_product(row, r.xq, beta, torch.float32),
                       dmmv.dmmv_block_product(row, r.xq, apart[1], torch.float32))


def test_rows_without_columns(gpu_device):
    from paper_2508_13437_amd import dmmv

    r = dmmv.dmmv_layernorm(torch.empty(300, 0, device=gpu_device), q=True, xq=True)
    assert r.y.shape == (300, 0) and torch.isnan(r.mean).all() and torch.isnan(r.rstd).all()


def test_no_rows_and_another_stream(gpu_device):
    from paper_2508_13437_amd import dmmv

    e = torch.empty(0, 40, device=gpu_device)
    r = dmmv.dmmv_layernorm(e, q=True)
    dx, dg, db = dmmv.dmmv_layernorm_backward(e, e, None, r.mean, r.rstd)
    assert dx.shape == (0, 40) and (dg == 0).all() and (db == 0).all()
    e = torch.empty(4, 0, device=gpu_device)
    assert dmmv.dmmv_layernorm(e).y.shape == (4, 0)
    x = make(50, 700, torch.bfloat16, 8, gpu_device)
    want = dmmv.dmmv_layernorm(x).y
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = dmmv.dmmv_layernorm(x).y
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    x = torch.randn(4, 200, device=gpu_device)
    g = torch.ones(200, device=gpu_device)
    r = dmmv.dmmv_layernorm(x, g, xq=True)
    for args, status in (((x.half(),), -3), ((x, g[:199]), -2), ((x, g.double()), -3), ((x, g, g, -1.0), -4), ((x, g, g, float("nan")), -4),
                         ((x.cpu(),), -6), ((x[0],), -2)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_layernorm(*args)
        assert e.value.status == status
    for args, status in (((x, x[:3], g, r.mean, r.rstd), -2), ((x, x.bfloat16(), g, r.mean, r.rstd), -3), ((x, x, g, r.mean[:2], r.rstd), -2),
                         ((x[:3], r.xq, g, r.mean[:3], r.rstd[:3]), -2)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_layernorm_backward(*args)
        assert e.value.status == status
    lib, s, p = dmmv.load(), torch.cuda.current_stream().cuda_stream, x.data_ptr()
    ws = torch.empty(lib.dmmv_layernorm_workspace_bytes(4, 200), dtype=torch.uint8, device=gpu_device)
    call = lambda w, n, x1, q1: lib.dmmv_layernorm_backward(dmmv.DMMV_F32, 4, 200, p, 200, x1, 200, q1, None, r.mean.data_ptr(),  # noqa: E731
                                                             r.rstd.data_ptr(), None, 0, g.data_ptr(), None, w, n, s)
    assert call(None, 0, p, None) == -5 and call(ws.data_ptr(), 8, p, None) == -5 and call(ws.data_ptr() + 4, 1 << 20, p, None) == -5
    assert call(ws.data_ptr(), ws.numel(), p, r.xq._p) == -1 and call(ws.data_ptr(), ws.numel(), None, None) == -1
    assert lib.dmmv_layernorm_workspace_bytes(-1, 5) == 0 and lib.dmmv_layernorm_workspace_bytes(5, 1 << 40) == 0
