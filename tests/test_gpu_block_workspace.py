"""The gradients with a workspace of exactly the bytes that the size function gives, between bytes that must stay."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def matrix(rows, K, kind, seed, device, pad):
    from paper_2508_13437_amd import dmmv

    r = np.random.default_rng(seed)
    codes = torch.from_numpy(r.integers(-8, 9, (rows, K + pad)).astype(np.float32)).to(device).to(torch.float8_e4m3fn)[:, pad:]
    nb = -(-K // 128)
    if kind == "e8m0":
        return dmmv.BlockMatrix(codes, torch.from_numpy(r.integers(125, 129, (rows, nb)).astype(np.uint8)).to(device))
    s = torch.from_numpy(2.0 ** r.integers(-2, 3, (rows, nb if kind == "f32" else 1)).astype(np.float32)).to(device)
    return dmmv.BlockMatrix(codes, s.expand(-1, nb))


# by the large tiles as they are and laid out, by the small ones with and without shares of the contraction, laid out; the bias in one step and two
@pytest.mark.parametrize("T,O,K", [(2048, 4096, 2048), (2050, 4101, 2051), (777, 1365, 1003), (64, 2050, 400), (2051, 66, 390), (1, 1024, 512), (3000, 40, 70), (9, 6, 300)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kx,kw", [("e8m0", "e8m0"), ("row", "row"), ("e8m0", "row"), ("f32", "f32")])
def test_workspace_of_the_least_size(gpu_device, T, O, K, dtype, kx, kw):
    from paper_2508_13437_amd import dmmv

    lib, name = dmmv.load(), dmmv.DMMV_F32 if dtype == torch.float32 else dmmv.DMMV_BF16
    for pad in (0, 1):
        x, w = matrix(T, K, kx, T, gpu_device, pad), matrix(O, K, kw, O, gpu_device, pad)
        dy = torch.from_numpy(np.random.default_rng(K).integers(-8, 9, (T, O + pad)).astype(np.float32)).to(dtype).to(gpu_device)[:, pad:]
        out = [torch.empty(s, dtype=d, device=gpu_device) for s, d in (((T, K), dtype), ((O, K), torch.float32), ((O,), torch.float32))]
        px, pw, pb = (t.data_ptr() for t in out)
        n = lib.dmmv_block_backward_workspace_for(name, T, O, K, dy.data_ptr(), dy.stride(0), x._p, w._p, px, pw)
        room = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device=gpu_device)
        at = -room.data_ptr() % 256 + 4096 - 4096 % 256
        stream = torch.cuda.current_stream().cuda_stream
        call = lambda bytes_: lib.dmmv_block_backward(name, T, O, K, dy.data_ptr(), dy.stride(0), x._p, w._p, px, K, pw, K, pb, room.data_ptr() + at, bytes_, stream)  # noqa: E731
        assert call(n - 1) == -5                             # refused before anything is enqueued
        dmmv._check(call(n))
        assert bool((room[:at] == 0xA5).all()) and bool((room[at + n:] == 0xA5).all())
        W, X, D = (dmmv.dmmv_block_dequantize(w, torch.float32).double(), dmmv.dmmv_block_dequantize(x, torch.float32).double(), dy.double())
        assert torch.equal(out[0], (D @ W).to(dtype))        # small integers: exact
        assert torch.equal(out[1].double(), D.t() @ X) and torch.equal(out[2].double(), D.sum(0))


@pytest.mark.parametrize("dtype,kind,pad,needs", [(torch.float32, "e8m0", 1, "nothing"), (torch.float32, "f32", 0, "nothing"), (torch.bfloat16, "f32", 1, "nothing"),
                                                  (torch.bfloat16, "e8m0", 1, "codes"), (torch.bfloat16, "row", 1, "codes")])
def test_a_product_needs_a_workspace_where_it_uses_one(gpu_device, dtype, kind, pad, needs):
    """A large product of unaligned rows: the codes are laid out for bf16 results with exponents, and nothing is for others."""
    from paper_2508_13437_amd import dmmv

    lib, name = dmmv.load(), dmmv.DMMV_F32 if dtype == torch.float32 else dmmv.DMMV_BF16
    T, O, K = 200, 4000, 8191
    x, w = matrix(T, K, kind, 1, gpu_device, pad), matrix(O, K, kind, 2, gpu_device, pad)
    y = torch.empty(T, O, dtype=dtype, device=gpu_device)
    most = lib.dmmv_block_product_workspace_bytes(T, O, K)
    lay = (T + O) * 8192
    assert most >= lay
    stream = torch.cuda.current_stream().cuda_stream
    call = lambda p, n: lib.dmmv_block_product(x._p, w._p, None, name, y.data_ptr(), O, p, n, stream)  # noqa: E731
    if needs == "nothing":
        dmmv._check(call(None, 0))
    else:
        assert call(None, 0) == -5
        room = torch.full((most + 4096,), 0xA5, dtype=torch.uint8, device=gpu_device)
        assert call(room.data_ptr(), lay - 1) == -5
        dmmv._check(call(room.data_ptr(), most))
        assert bool((room[most:] == 0xA5).all())
    want = dmmv.dmmv_block_dequantize(x, torch.float32).double() @ dmmv.dmmv_block_dequantize(w, torch.float32).double().t()
    assert torch.equal(y, want.to(dtype)) and torch.equal(dmmv.dmmv_block_product(x, w, dtype=dtype), y)
