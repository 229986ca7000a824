"""A BlockMatrix stands for the memory it was made of, whatever becomes of the tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def make(rows, cols, device):
    g = torch.Generator().manual_seed(rows)
    return (torch.randint(0x30, 0x40, (rows, cols), generator=g, dtype=torch.uint8).to(device),
            torch.randint(120, 130, (rows, -(-cols // 128)), generator=g, dtype=torch.uint8).to(device))


def test_sizes_and_tensors_are_fixed(gpu_device):
    from paper_2508_13437_amd import dmmv

    codes, scales = make(6, 300, gpu_device)
    for q in (dmmv.BlockMatrix(codes, scales), dmmv.dmmv_block_quantize(torch.randn(6, 300, device=gpu_device))):
        for name, value in (("codes", codes[:3]), ("scales", scales * 0), ("scale_rows", 128), ("rows", 5), ("cols", 200)):
            with pytest.raises(AttributeError):
                setattr(q, name, value)
        assert (q.rows, q.cols, q.scale_rows, q.device) == (6, 300, 1, codes.device)
        assert q.codes.shape == (6, 300) and q.scales.shape == (6, 3) and q.values8.dtype == torch.float8_e4m3fn


def test_numbers_written_are_seen_and_other_tensors_are_not(gpu_device):
    from paper_2508_13437_amd import dmmv

    codes, scales = make(6, 300, gpu_device)
    w = dmmv.BlockMatrix(*make(70, 300, gpu_device))
    q = dmmv.BlockMatrix(codes, scales)
    f = dmmv.BlockMatrix(q.values8, scales)                 # the same memory as float8
    first = dmmv.dmmv_block_product(q, w, dtype=torch.float32)
    scales.add_(1)                                           # in place: twice the values
    assert torch.equal(dmmv.dmmv_block_product(q, w, dtype=torch.float32), 2.0 * first)
    q.scales.sub_(1)
    q.codes[3] = 0
    first[3] = 0.0
    assert torch.equal(dmmv.dmmv_block_product(q, w, dtype=torch.float32), first)
    # the tensors get other memory: what the matrix stands for stays, and stays allocated
    codes.data, scales.data = torch.zeros(2, 2, dtype=torch.uint8, device=gpu_device), torch.zeros(1, 1, dtype=torch.uint8, device=gpu_device)
    q.codes.set_(codes)
    q.scales.set_(scales)
    f.values8.set_(codes.view(torch.float8_e4m3fn))
    del codes, scales
    junk = [torch.full((6, 300), 0x7F, dtype=torch.uint8, device=gpu_device) for _ in range(8)]
    assert all(torch.equal(dmmv.dmmv_block_product(m, w, dtype=torch.float32), first) for m in (q, f)) and len(junk) == 8
    assert torch.equal(dmmv.dmmv_block_dequantize(q, torch.float32)[3], torch.zeros(300, device=gpu_device))


def test_codes_whose_rows_are_not_contiguous_are_copied(gpu_device):
    from paper_2508_13437_amd import dmmv

    codes, scales = make(6, 300, gpu_device)
    turned = codes.t().contiguous().t()
    a, b = dmmv.BlockMatrix(codes, scales), dmmv.BlockMatrix(turned, scales)
    turned.zero_()
    w = dmmv.BlockMatrix(*make(70, 300, gpu_device))
    assert torch.equal(dmmv.dmmv_block_product(a, w), dmmv.dmmv_block_product(b, w))
