"""The product's epilogue where scales are beyond what the tiles' loop takes and results are made once more: more than 64 tokens, 32-bit results or
32-bit scales.  A shift of x's scales against w's leaves every product as it is, so sums are exact still."""
import ctypes as C

import pytest
import torch

from tests import residual_plain as rp
from tests.test_gpu_block_linear import check, operands

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# exponents: bytes 1 and 2 of x (w at 244 and more), 2 and 3 of w; floats from 2^-126 on and up to 2^101
CASES = [("e8m0", "e8m0", -125, [F32]), ("e8m0", "e8m0", 117, [F32]), ("e8m0", "row", -125, [F32]), ("f32", "f32", -125, [F32, BF16]), ("f32", "f32", -100, [F32, BF16]),
         ("f32", "f32", 100, [F32, BF16])]


def shifted(q, by, blocks):
    """The scales times 2^by in some blocks of columns."""
    from paper_2508_13437_amd import dmmv

    if q.scales.dtype == torch.uint8:
        s = torch.where(blocks, q.scales.int() + by, q.scales.int())
        assert 1 <= int(s.min()) and int(s.max()) <= 254
        return dmmv.BlockMatrix(q.codes, s.to(torch.uint8), q.scale_rows)
    if q.scales.stride(1) == 0:                                             # one for the row
        return dmmv.BlockMatrix(q.codes, (q.scales[:, :1] * 2.0 ** by).expand(-1, q.scales.shape[1]), 1)
    return dmmv.BlockMatrix(q.codes, torch.where(blocks, q.scales * 2.0 ** by, q.scales), q.scale_rows)


def far_operands(T, O, K, kx, kw, by, g, some, device):
    x, w, bias, want = operands(T, O, K, kx, kw, device, g)
    blocks = torch.arange(x.scales.shape[1], device=device)[None] % 3 != 1 if some and kw != "row" else torch.ones(1, x.scales.shape[1], dtype=torch.bool, device=device)
    return shifted(x, by, blocks), shifted(w, -by, blocks), bias, want


@pytest.mark.parametrize("kx,kw,by,types", CASES)
@pytest.mark.parametrize("T,O,K", [(70, 140, 300), (300, 130, 521), (65, 64, 128), (129, 257, 1000)])
def test_linear(gpu_device, T, O, K, kx, kw, by, types):
    from paper_2508_13437_amd import dmmv

    for g, some in ((1, True), (128, True), (128, False)) if kw == "e8m0" else ((None, True), (None, False)):
        x, w, bias, want = far_operands(T, O, K, kx, kw, by, g, some, gpu_device)
        gen = torch.Generator().manual_seed(T * O)
        for i, kind in enumerate((None, *rp.ACTS)):
            for dtype in types:
                res = torch.randn(T, O + 3, generator=gen).to(dtype).to(gpu_device)[:, 3:] if i % 2 == 0 else None
                r = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=True, q=True, u=True)
                check(r, want, kind, res, dtype, dtype == BF16)
                if dtype == F32:
                    q = dmmv.dmmv_block_quantize(r.y)
                    assert torch.equal(q.codes, r.q.codes) and torch.equal(q.scales, r.q.scales)
                only = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=False, q=True)
                assert torch.equal(only.q.codes, r.q.codes) and torch.equal(only.q.scales, r.q.scales)
                only = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, u=True)
                check(only, want, kind, res, dtype, dtype == BF16)
                assert torch.equal(only.u, r.u) and torch.equal(only.u, dmmv.dmmv_block_product(x, w, bias, dtype))


@pytest.mark.parametrize("kx,kw,by,types", [CASES[0], CASES[3]])
def test_rows_with_gaps(gpu_device, kx, kw, by, types):
    """Through the C entry: rows wider than the results; what lies between them stays as it was."""
    from paper_2508_13437_amd import dmmv

    lib, T, O = dmmv.load(), 130, 141
    x, w, bias, _ = far_operands(T, O, 300, kx, kw, by, 128 if kw == "e8m0" else None, True, gpu_device)
    for dtype in types:
        code = dmmv.DMMV_F32 if dtype == F32 else dmmv.DMMV_BF16
        res = torch.randn(T, O + 1, device=gpu_device).to(dtype)
        want = dmmv.dmmv_block_linear(x, w, bias, "gelu", res[:, :O], dtype, q=True, u=True)
        y, u = (torch.full((T + 1, O + 5), 7.0, dtype=dtype, device=gpu_device) for _ in range(2))
        codes, scales = torch.full((T + 1, O + 3), 77, dtype=torch.uint8, device=gpu_device), torch.full((T + 1, 4), 66, dtype=torch.uint8, device=gpu_device)
        q = dmmv._BlockMatrix(T, O, codes.data_ptr(), O + 3, scales.data_ptr(), 4, 1, dmmv.DMMV_E8M0, 1)
        n = lib.dmmv_block_linear_workspace_for(x._p, w._p, code, 1)
        ws = torch.empty(n, dtype=torch.uint8, device=gpu_device)
        s = lib.dmmv_block_linear(x._p, w._p, bias.data_ptr(), 2, res.data_ptr(), O + 1, code, y.data_ptr(), O + 5, C.addressof(q), u.data_ptr(), O + 5, ws.data_ptr(), n,
                                  torch.cuda.current_stream().cuda_stream)
        assert s == 0, lib.dmmv_last_error()
        for got, one in ((y, want.y), (u, want.u), (codes, want.q.codes.view(torch.uint8)), (scales, want.q.scales)):
            assert torch.equal(got[:T, :one.shape[1]], one)
            rest = got.clone()
            rest[:T, :one.shape[1]] = got[T, -1]
            assert bool((rest == got[T, -1]).all())
