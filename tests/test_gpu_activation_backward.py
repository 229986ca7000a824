"""Back through an activation, and the gradient of the bias, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import residual_plain as rp
from tests.test_gpu_block_product import f64, half_ulp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 1), (1, 4096), (3, 7), (9, 96), (50, 128), (700, 130), (33, 512), (1025, 513), (5, 2049), (513, 1003), (3000, 70), (257, 11008)]


def make(rows, cols, dtype, seed, device, pad=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(rows, cols + pad, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype).to(device)[:, pad:]


def slope_error(u, kind):
    """Of the derivative of an exact u.  The logistic's argument has at most six roundings (its exponential's error is that times it), the
    products and sums of s + u s (1 - s) x' ten; erfc is within 32 U of itself, its argument two roundings; the density's
    argument three, its exponential two and four products."""
    if kind == "relu":
        return 0.0 * u
    a = np.minimum(np.abs(u), 30.0)
    if kind == "gelu":
        area = 0.5 * rp.erfc(-u / np.sqrt(2.0))
        density = a * np.exp(-a * a / 2.0) / np.sqrt(2.0 * np.pi)
        return ((2 * (a * a + 2 * a) + 36) * area + (3 * a * a + 12) * density) * U + 1e-36
    x, grow = (np.abs(u), 1.0) if kind == "silu" else (np.abs(2.0 * rp.K * (u + 0.044715 * u ** 3)), 2.0 * rp.K * (1.0 + 3 * 0.044715 * u ** 2))
    s, t = rp.expit(np.sign(u) * x), rp.expit(-np.sign(u) * x)
    k = 6 * np.minimum(x, 200.0) + 14
    return (k * s + (2 * k + 10) * np.abs(u) * s * t * grow) * U + 1e-35


@pytest.mark.parametrize("kind", rp.ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(gpu_device, rows, cols, dtype, kind):
    from paper_2508_13437_amd import dmmv

    for pad in (0, 1):
        dy, u = make(rows, cols, dtype, rows, gpu_device, pad, 0.01), make(rows, cols, dtype, cols, gpu_device, 3 * pad)
        du, db = dmmv.dmmv_activation_backward(dy, u, kind)
        d, want = f64(dy), rp.slope(f64(u), kind)
        # below 2^-126 a rounding is absolute: half of the type's smallest number, 2^-133 or 2^-149
        e = np.abs(d) * (slope_error(f64(u), kind) + U * np.abs(want)) * 1.01 + (2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -149)
        want = d * want
        assert (np.abs(f64(du) - want) <= e + half_ulp(dtype) * 1.01 * (np.abs(want) + e)).all()
        # at most `rows` additions one after another
        assert (np.abs(f64(db) - want.sum(0)) <= e.sum(0) + (rows + 20) * U * np.abs(want).sum(0)).all()
        again = dmmv.dmmv_activation_backward(dy, u, kind)
        assert torch.equal(again[0], du) and torch.equal(again[1], db)
        only = dmmv.dmmv_activation_backward(dy, u, kind, du=False), dmmv.dmmv_activation_backward(dy, u, kind, dbias=False)
        assert only[0][0] is None and torch.equal(only[0][1], db) and only[1][1] is None and torch.equal(only[1][0], du)


def test_both_ends(gpu_device):
    from paper_2508_13437_amd import dmmv

    inf, nan = float("inf"), float("nan")
    u = torch.tensor([[0.0, -0.0, -1e-30, 1e-30, -20.0, 20.0, -110.0, 110.0, -1e20, 1e20, -3e38, 3e38, -inf, inf, nan]], device=gpu_device)
    for kind in rp.ACTS:
        got = f64(dmmv.dmmv_activation_backward(torch.ones_like(u), u, kind)[0])[0]
        half = 0.0 if kind == "relu" else 0.5
        assert np.isnan(got[-1]) and np.isfinite(got[:-1]).all()
        assert got[0] == got[1] == half and abs(got[2] - half) < 1e-7 and got[3] == (1.0 if kind == "relu" else 0.5)
        assert (np.abs(got[[6, 8, 10, 12]]) < 1e-30).all() and (got[[7, 9, 11, 13]] == 1.0).all()
        assert abs(got[4]) < 1e-7 and abs(got[5] - 1.0) < 1e-7
    dy = torch.zeros(3, 40, device=gpu_device)
    dy[1, 3], dy[2, 5] = inf, nan
    du, db = dmmv.dmmv_activation_backward(dy, torch.ones_like(dy), "gelu")
    assert float(du[1, 3]) == inf and du[2, 5].isnan() and du.isfinite().sum() == 118 and float(db[3]) == inf and db[5].isnan() and db.isfinite().sum() == 38


def test_no_rows_no_columns_and_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    e = torch.empty(0, 40, device=gpu_device)
    du, db = dmmv.dmmv_activation_backward(e, e, "silu")
    assert du.shape == (0, 40) and (db == 0).all()
    e = torch.empty(4, 0, device=gpu_device)
    du, db = dmmv.dmmv_activation_backward(e, e, "silu")
    assert du.shape == (4, 0) and db.shape == (0,)
    x = torch.randn(4, 20, device=gpu_device)
    for args, status in (((x, x, None), -4), ((x, x, "tanh"), -4), ((x, x[:3], "relu"), -2), ((x, x.bfloat16(), "relu"), -3), ((x.half(), x.half(), "relu"), -3),
                         ((x, x.cpu(), "relu"), -6), ((x[0], x[0], "relu"), -2)):
        with pytest.raises(dmmv.DmmvError) as err:
            dmmv.dmmv_activation_backward(*args)
        assert err.value.status == status
    # transposed inputs are copied, in the order that the call reads
    a, b = torch.randn(30, 20, device=gpu_device), torch.randn(30, 20, device=gpu_device)
    want = dmmv.dmmv_activation_backward(a.t().contiguous(), b.t().contiguous(), "gelu")
    got = dmmv.dmmv_activation_backward(a.t(), b.t(), "gelu")
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_row_of_more_pieces_than_a_grid_is_high(gpu_device):
    """65537 pieces of 2048 columns.  max(u, 0): the gradient is dy itself or 0."""
    from paper_2508_13437_amd import dmmv

    cols = 65536 * 2048 + 5
    dy = torch.arange(cols, device=gpu_device, dtype=torch.int32).remainder_(251).to(torch.bfloat16)[None] + 1
    u = torch.where(torch.arange(cols, device=gpu_device, dtype=torch.int32).remainder_(3) == 0, -1.0, 1.0).to(torch.bfloat16)[None]
    du, db = dmmv.dmmv_activation_backward(dy, u, "relu", dbias=False)
    assert db is None and torch.equal(du, torch.where(u > 0, dy, torch.zeros_like(dy)))
