"""How far activations and their derivatives may be off in 32 bits, over the whole range in which they do not vanish.

Units of 2^-24.  Of the functions of the hardware, 2^x and 1 / x, a result is off by one in the last place, 2 units.
    u Phi(u): t^2 / 2 in the exponent has two roundings and a constant's 0.22, times t^2 / 2: 1.11 t^2; 2^x 2; the polynomial 5.6, its variable 3 (1 / x, a
    sum), of which the quotient makes up to 8 / 3 times as much; three products
    logistic of x: the product with log2 e one rounding and a constant's 0.22, times |x|: 1.22 |x|; 2^x 2, the sum 1, 1 / x 2, two products
    its x = 2 z: constants 0.48 and 0.58, products and a sum 5, times |x|, beside log2 e: 7.3 |x| at most
A derivative has those errors in its two terms, in the second once for each factor, and five products and sums.  2^x has no results below 2^-126: what
is smaller than 230 times that may be lost.
"""
import numpy as np
import pytest
import torch

from tests import residual_plain as rp
from tests.test_gpu_block_product import f64

pytestmark = pytest.mark.gpu
UNIT, LOST = 2.0 ** -24, 2.0 ** -118


def grid(device):
    u = np.concatenate([np.linspace(-110.0, 110.0, 300001), np.linspace(-14.0, 2.0, 100001), *(s * np.exp(np.linspace(-60.0, 1.0, 20000)) for s in (-1, 1))])
    return torch.from_numpy(u.astype(np.float32)).to(device)


def units(u, kind):
    z = np.abs(rp.K * (u + 0.044715 * u ** 3))
    return {"relu": 0.0 * u, "gelu": 1.2 * u * u + 20.0, "gelu_tanh": 15.0 * z + 8.0, "silu": 1.3 * np.abs(u) + 8.0}[kind]


def terms(u, kind):
    """The magnitudes of a derivative's two terms."""
    if kind == "relu":
        return (u > 0).astype(np.float64), 0.0 * u
    if kind == "gelu":
        return 0.5 * rp.erfc(-u / np.sqrt(2.0)), np.abs(u) * np.exp(-u * u / 2.0) / np.sqrt(2.0 * np.pi)
    x, grow = (u, 1.0) if kind == "silu" else (2.0 * rp.K * (u + 0.044715 * u ** 3), 2.0 * rp.K * (1.0 + 3 * 0.044715 * u ** 2))
    return rp.expit(x), np.abs(u) * rp.expit(x) * rp.expit(-x) * grow


@pytest.mark.parametrize("kind", rp.ACTS)
def test_activation(gpu_device, kind):
    """u by the bias: the product is 0."""
    from paper_2508_13437_amd import dmmv

    u = grid(gpu_device)
    for T in (1, 70):
        x, w = (dmmv.BlockMatrix(torch.zeros(n, 128, dtype=torch.uint8, device=gpu_device)) for n in (T, len(u)))
        want = rp.act(f64(u), kind)
        got = f64(dmmv.dmmv_block_linear(x, w, u, kind, dtype=torch.float32).y)
        assert (np.abs(got - want) <= units(f64(u), kind) * UNIT * np.abs(want) + LOST).all()
        got = f64(dmmv.dmmv_block_linear(x, w, u, kind).y)
        assert (np.abs(got - want) <= (2.0 ** -14 + 2.0 ** -8 * 1.001) * np.abs(want) + LOST).all()


@pytest.mark.parametrize("kind", rp.ACTS)
def test_derivative(gpu_device, kind):
    from paper_2508_13437_amd import dmmv

    u = grid(gpu_device)[None]
    got = f64(dmmv.dmmv_activation_backward(torch.ones_like(u), u, kind, dbias=False)[0])
    e = (2.0 * units(f64(u), kind) + 20.0) * UNIT * sum(terms(f64(u), kind))
    assert (np.abs(got - rp.slope(f64(u), kind)) <= e + LOST).all()
