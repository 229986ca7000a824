"""Values of 8-bit matrices with 32-bit scales: rounded once."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu


def nearest(v, bits, low, top):
    """float64 to the nearest number of `bits` significant bits, ties to even, multiples of 2^low at least, infinite from 2^top on."""
    with np.errstate(invalid="ignore"):
        e = np.frexp(np.where(np.isfinite(v) & (v != 0), v, 1.0))[1]
        step = np.ldexp(1.0, np.maximum(e - bits, low))
        r = np.rint(v / step) * step
    return np.where(np.isfinite(v) & (np.abs(r) >= 2.0 ** top), np.copysign(np.inf, v), np.where(np.isfinite(v), r, v))


@pytest.mark.parametrize("exponents", [(-3, 3), (-149, -120), (115, 128), (-140, 128)])
def test_values_are_rounded_once(gpu_device, exponents):
    """Every code with scales of 24 bits: 28 bits before the rounding, to bf16 and to 32 bits."""
    from paper_2508_13437_amd import dmmv

    r = np.random.default_rng(exponents[1] + 200)
    rows, blocks = 512, 40
    with np.errstate(over="ignore"):
        s = np.ldexp(r.uniform(0.5, 1.0, (rows, blocks)), r.integers(exponents[0], exponents[1] + 1, (rows, blocks))).astype(np.float32)
    s *= r.choice([-1.0, 1.0], s.shape).astype(np.float32)
    s[0, 0], s[0, 1] = np.float32(float.fromhex("0x1.f95554p+0")), 0.0
    codes = np.resize(r.permutation(256).astype(np.uint8), (rows, blocks * 128 - 3))
    codes[0, :128] = 0x06                                    # 0.01171875
    q = dmmv.BlockMatrix(torch.from_numpy(codes).to(gpu_device), torch.from_numpy(s).to(gpu_device))
    v = plain.values(codes, s)                               # exact
    for dtype, want in ((torch.bfloat16, nearest(v, 8, -133, 128)), (torch.float32, nearest(v, 24, -149, 128))):
        got = dmmv.dmmv_block_dequantize(q, dtype).double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)
    if exponents == (-3, 3):
        assert float(dmmv.dmmv_block_dequantize(q)[0, 0]) == 0.0230712890625


def test_values_of_scales_that_are_not_finite(gpu_device):
    from paper_2508_13437_amd import dmmv

    codes = torch.tensor([[0x38, 0xB8, 0x00, 0x7F]], dtype=torch.uint8, device=gpu_device).expand(2, -1).contiguous()
    q = dmmv.BlockMatrix(codes, torch.tensor([[float("inf")], [float("nan")]], device=gpu_device))
    for dtype in (torch.bfloat16, torch.float32):
        got = dmmv.dmmv_block_dequantize(q, dtype).float().cpu().numpy()
        assert np.array_equal(got, np.array([[np.inf, -np.inf, np.nan, np.nan], [np.nan] * 4], np.float32), equal_nan=True)
