"""Matrices in 8 bits: codes and scales against the definition, bit for bit; values back, bit for bit."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (1, 7), (2, 8), (1, 127), (3, 128), (5, 129), (16, 130), (130, 257), (129, 1000), (40, 2731), (1, 11008)]


def make(rows, cols, dtype, seed, device, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + pad, generator=g) * torch.exp(3.0 * torch.randn(rows, 1, generator=g))
    x = torch.where(torch.rand(rows, cols + pad, generator=g) < 0.01, x * 1e4, x).to(dtype)
    return x.to(device)[:, pad:]                              # pad > 0: rows with a stride, off by one element


def check(x, q, g):
    from paper_2508_13437_amd import dmmv

    want_c, want_s = plain.quantize(x.double().cpu().numpy(), g)
    got_s = q.scales.cpu().numpy()
    if got_s.dtype == np.float32:
        assert np.array_equal(got_s.astype(np.float64), plain.scale_values(want_s))
    else:
        assert np.array_equal(got_s, want_s)
    assert np.array_equal(q.codes.cpu().numpy(), want_c)
    for dtype in (torch.float32, torch.bfloat16):
        back = dmmv.dmmv_block_dequantize(q, dtype).float().cpu().numpy()
        want = torch.from_numpy(plain.values(want_c, want_s, g)).to(dtype).float().numpy()
        assert np.array_equal(back, want, equal_nan=True)


@pytest.mark.parametrize("g", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_scales_and_values(gpu_device, rows, cols, dtype, g):
    from paper_2508_13437_amd import dmmv

    for pad in (0, 1):
        x = make(rows, cols, dtype, 100 * rows + cols, gpu_device, pad)
        check(x, dmmv.dmmv_block_quantize(x, g, torch.uint8 if pad else torch.float32), g)


@pytest.mark.parametrize("g", [1, 128])
def test_zeros_extremes_and_what_is_not_finite(gpu_device, g):
    from paper_2508_13437_amd import dmmv

    x = torch.randn(7, 300, generator=torch.Generator().manual_seed(5))
    x[0] = 0.0                                   # a block of zeros: scale 1
    x[1] *= 1e-42                                # denormal numbers: the smallest scale
    x[2, :128] *= 3e38 / x[2, :128].abs().max()  # the largest scale
    x[3, 5], x[3, 140], x[3, 299] = float("nan"), float("inf"), float("-inf")
    x[4] = float("nan")                          # nothing finite in the block
    x[5, :128] = 448.0                           # the edge of a scale, and just over it
    x[5, 130:260] = float(np.nextafter(np.float32(448.0), np.float32(500.0)))
    x[6] = -0.0
    x = x.to(gpu_device)
    check(x, dmmv.dmmv_block_quantize(x, g), g)


def test_halfway_values_go_to_the_even_code(gpu_device):
    from paper_2508_13437_amd import dmmv

    mid = torch.from_numpy((plain.E4M3[:126] + plain.E4M3[1:127]) / 2).float()
    x = torch.cat([mid, torch.tensor([448.0, 1.0])])[None].repeat(2, 1)
    x[1] *= -(2.0 ** -20)
    x = x.to(gpu_device)
    check(x, dmmv.dmmv_block_quantize(x), 1)


def test_scale_strides_and_long_row_strides(gpu_device):
    """Codes with rows 2^31 bytes apart (offsets past 32 bits) and scales stored block by block."""
    import ctypes as C

    from paper_2508_13437_amd import dmmv

    x = make(3, 300, torch.float32, 9, gpu_device)
    ld = (1 << 31) + 24
    buf = torch.empty(2 * ld + 300, dtype=torch.uint8, device=gpu_device)
    codes = buf.as_strided((3, 300), (ld, 1))
    scales = torch.zeros(3, 3, dtype=torch.uint8, device=gpu_device).t()
    q = dmmv.BlockMatrix(codes, scales)
    dmmv._check(dmmv.load().dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr(), x.stride(0), q._p,
                                                C.c_void_p(torch.cuda.current_stream().cuda_stream)))
    check(x, q, 1)


def test_empty(gpu_device):
    from paper_2508_13437_amd import dmmv

    for shape in ((0, 5), (4, 0), (0, 0)):
        q = dmmv.dmmv_block_quantize(torch.empty(shape, device=gpu_device))
        assert dmmv.dmmv_block_dequantize(q).shape == shape


def test_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    x = torch.randn(4, 200, device=gpu_device)
    for bad, status in ((x.double(), -3), (x[0], -2), (x.cpu(), -6)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_block_quantize(bad)
        assert e.value.status == status
    q = dmmv.dmmv_block_quantize(x)
    for codes, scales, g, status in ((q.codes.float(), None, 1, -3), (q.codes, q.scales[:, :1], 1, -2), (q.codes, None, 64, -2),
                                     (q.codes, q.scales.double(), 1, -3), (q.codes.cpu(), None, 1, -6)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.BlockMatrix(codes, scales, g)
        assert e.value.status == status
    lib, s = dmmv.load(), torch.cuda.current_stream().cuda_stream
    good = dmmv.BlockMatrix(torch.zeros(4, 200, dtype=torch.uint8, device=gpu_device), torch.zeros(4, 2, dtype=torch.uint8, device=gpu_device))
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr(), 199, good._p, s) == -2          # stride below the columns
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr() + 2, 200, good._p, s) == -2      # not aligned to its elements
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, None, 200, good._p, s) == -1
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr(), 200, None, s) == -1
    assert lib.dmmv_block_quantize(dmmv.DMMV_F64, x.data_ptr(), 200, good._p, s) == -3
    shared = dmmv.BlockMatrix(good.codes, good.scales[:, :1].expand(-1, 2))                     # an output's scales may not overlap
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr(), 200, shared._p, s) == -2
    bare = dmmv.BlockMatrix(good.codes)
    assert lib.dmmv_block_quantize(dmmv.DMMV_F32, x.data_ptr(), 200, bare._p, s) == -1
