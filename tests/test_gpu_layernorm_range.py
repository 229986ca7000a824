"""Layer norm's gradient where mean * rstd is beyond the range: what is finite stays finite."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("from_8bit", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(3, 5), (2, 7), (6, 301), (600, 301), (5, 1003), (3, 4095), (2, 8191), (3, 8195), (2, 16390)])
def test_gradient_of_rows_without_variance_far_from_zero(gpu_device, rows, cols, dtype, from_8bit):
    """Every number 2^110 (or a power near it): h is 0, and dx = rstd (a - mean a)."""
    from paper_2508_13437_amd import dmmv

    g = torch.Generator().manual_seed(cols)
    x = (2.0 ** torch.randint(108, 112, (rows, 1), generator=g)).expand(-1, cols).to(dtype).contiguous().to(gpu_device)
    dy = torch.randn(rows, cols, generator=g).to(dtype).to(gpu_device)
    gamma = (1.0 + 0.2 * torch.randn(cols, generator=g)).to(gpu_device)
    r = dmmv.dmmv_layernorm(x, gamma, None, 1e-12, y=True, xq=True)
    assert torch.equal(r.mean, x[:, 0].float()) and bool((r.y == 0).all())
    dx, dgamma, dbeta = (t.double().cpu().numpy() for t in dmmv.dmmv_layernorm_backward(dy, r.xq if from_8bit else x, gamma, r.mean, r.rstd))
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = plain.norm_grad(f64(dy), f64(x), f64(gamma), f64(r.mean), f64(r.rstd))
    a = np.abs(f64(dy) * f64(gamma))
    # a row's sums: a lane's own terms one after the other and a tree of at most 1024 lanes; the formula's five more
    n = 8 * max(1, -(-cols // 2048)) + 26
    e = f64(r.rstd)[:, None] * (a + a.mean(1, keepdims=True)) * (n + 8) * U
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    assert (np.abs(dx - want[0]) <= e + half * 1.01 * (np.abs(want[0]) + e)).all()
    assert (dgamma == 0).all() and (np.abs(dbeta - want[2]) <= (rows + 20) * U * np.abs(f64(dy)).sum(0)).all()


def test_missing_arguments_are_refused(gpu_device):
    from paper_2508_13437_amd import dmmv

    x = torch.randn(4, 200, device=gpu_device)
    r = dmmv.dmmv_layernorm(x, xq=True)
    for args in ((x, None, None, r.mean, r.rstd), (x, x, None, None, r.rstd), (x, r.xq, None, r.mean, None)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_layernorm_backward(*args)
        assert e.value.status == -1
