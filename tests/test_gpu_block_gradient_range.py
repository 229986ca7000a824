"""Gradients where exponents come near the ends of bf16's range, in every form that makes them."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# the large tiles (bf16) and dy laid out for them, small tiles with dy laid out (32 bits), the general form, shares of the contraction, short rows
SIZES = [(1024, 4096, 2048), (777, 1365, 1003), (150, 140, 300), (9, 2050, 70), (64, 64, 3)]


def codes_of(rows, K, seed, device):
    c = np.random.default_rng(seed).integers(0, 254, (rows, K)).astype(np.uint8)
    return torch.from_numpy(np.where(c & 127 == 127, 1, c).astype(np.uint8)).to(device)


def matrix(rows, K, byte, seed, device, pad=0):
    from paper_2508_13437_amd import dmmv

    b = torch.full((rows, -(-K // 128)), byte, dtype=torch.uint8, device=device)
    return dmmv.BlockMatrix(codes_of(rows, K + pad, seed, device)[:, pad:], b)


def values(q):
    return torch.from_numpy(plain.values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.scale_rows)).to(q.device)


def gradient(T, O, dtype, exponent, seed, device):
    r = np.random.default_rng(seed)
    return torch.from_numpy(np.ldexp(r.standard_normal((T, O)), exponent).astype(np.float32)).to(dtype).to(device)


def check(got, want, size, n, dtype, more=0.0):
    """Sums of n products of numbers of 24 bits at most (a bf16 result may come from 16); `more`: what else a result may be off by."""
    e = ((n + 12) * 2 * U + (2.0 ** -15 if dtype == torch.bfloat16 else 0.0)) * size + more
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    assert bool(torch.isfinite(got).all())
    assert bool(((got.double() - want).abs() <= e + half * 1.01 * (want.abs() + e)).all())


@pytest.mark.parametrize("T,O,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 246])
def test_exponents_at_the_ends(gpu_device, T, O, K, dtype, byte):
    """Bytes 3 to 246 are exact; below, a value is the nearest multiple of 2^-133."""
    from paper_2508_13437_amd import dmmv

    for pad in (0, 1) if T * O < 1e6 else (0,):
        x, w = matrix(T, K, byte, T, gpu_device, pad), matrix(O, K, byte, O, gpu_device, pad)
        dy = gradient(T, O, dtype, 60 if byte < 100 else -60, K, gpu_device)
        X, W, D = values(x), values(w), dy.double()
        dx, dw, _ = dmmv.dmmv_block_backward(dy, x, w)
        off = 2.0 ** -134 * 1.01 if byte < 3 else 0.0
        check(dx, D @ W, D.abs() @ W.abs(), O, dtype, off * D.abs().sum(1, keepdim=True))
        check(dw, D.t() @ X, D.t().abs() @ X.abs(), T, torch.float32, off * D.t().abs().sum(1, keepdim=True))


@pytest.mark.parametrize("T,O,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_exponent_byte_255(gpu_device, T, O, K, dtype):
    """NaN in the columns of its block, and nowhere else."""
    from paper_2508_13437_amd import dmmv

    x, w = matrix(T, K, 127, T, gpu_device), matrix(O, K, 127, O, gpu_device)
    dy = gradient(T, O, dtype, 0, K, gpu_device)
    want = dmmv.dmmv_block_backward(dy, x, w)
    last = (K - 1) // 128
    w.scales[O - 1, last], x.scales[T // 2, 0] = 255, 255
    dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
    assert bool(torch.isnan(dx[:, last * 128:]).all()) and torch.equal(dx[:, :last * 128], want[0][:, :last * 128])
    assert bool(torch.isnan(dw[:, :128]).all()) and torch.equal(dw[:, 128:], want[1][:, 128:]) and torch.equal(db, want[2])


@pytest.mark.parametrize("T,O,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["row", "f32"])
def test_small_32_bit_scales_keep_their_bits(gpu_device, T, O, K, dtype, kind):
    """Scales about 2^-95 and gradients about 1: what the gradients are made of is 2^-110 and more where it counts (a multiple of 2^-133 below)."""
    from paper_2508_13437_amd import dmmv

    def of(rows, seed):
        nb = -(-K // 128)
        s = np.ldexp(np.random.default_rng(seed).uniform(1.0, 2.0, (rows, nb if kind == "f32" else 1)), -95).astype(np.float32)
        return dmmv.BlockMatrix(codes_of(rows, K, seed, gpu_device), torch.from_numpy(s).to(gpu_device).expand(-1, nb))
    x, w = of(T, T), of(O, O)
    dy = gradient(T, O, dtype, 0, K, gpu_device)
    X, W, D = values(x), values(w), dy.double()
    dx, dw, _ = dmmv.dmmv_block_backward(dy, x, w)
    # three parts each cut at a multiple of 2^-133, of dy times a scale (times a code, 448 at most) or of a value (times dy)
    off = 2.0 ** -133 * 2.0
    check(dx, D @ W, D.abs() @ W.abs(), O, dtype, off * (D.abs().sum(1, keepdim=True) + 448.0 * O))
    check(dw, D.t() @ X, D.t().abs() @ X.abs(), T, torch.float32, off * (D.t().abs().sum(1, keepdim=True) + 448.0 * T))
