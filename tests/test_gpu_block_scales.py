"""Products of 8-bit matrices whose scales are far apart: what is finite stays finite and keeps its bits."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def codes_of(rows, K, seed, device):
    r = np.random.default_rng(seed)
    v = np.clip(r.standard_t(4.0, (rows, K)).astype(np.float32) * 20.0, -448, 448)
    return torch.from_numpy(v).to(device).to(torch.float8_e4m3fn)


def values(q):
    """A block matrix in 64 bits, on its device."""
    return torch.from_numpy(plain.values(q.codes.view(torch.uint8).cpu().numpy(), None if q.scales is None else q.scales.cpu().numpy(),
                                         q.scale_rows)).to(q.device)


def check_product(x, w, dtype, bias=None):
    from paper_2508_13437_amd import dmmv

    X, W, K = values(x), values(w), x.cols
    want, size = X @ W.t(), X.abs() @ W.abs().t()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    got = dmmv.dmmv_block_product(x, w, bias, dtype).double()
    # a sum of K exact products, three roundings for scales; bf16: what the 8-bit instructions drop, and the result's 8 bits
    e, half = (K + 8) * 2 * U * size, U
    if dtype == torch.bfloat16:
        e, half = e + 2.0 ** -10 * size, 2.0 ** -8
    assert bool(torch.isfinite(got).all())
    assert bool(((got - want).abs() <= e + half * 1.01 * (want.abs() + e)).all())
    assert float((got - want).norm()) <= (2e-6 + 1.01 * half) * float(want.norm()) + 1e-6 * float(size.norm()) / K ** 0.5


def powers(rows, blocks, exponent, seed, device):
    """Scales of 24 bits around 2^exponent (subnormal ones are exact multiples of 2^-149)."""
    r = np.random.default_rng(seed)
    s = np.ldexp(r.uniform(1.0, 1.9, (rows, blocks)), r.integers(exponent, exponent + 2, (rows, blocks)))
    return torch.from_numpy(s.astype(np.float32)).to(device)


APART = [(100, -100), (-100, 100), (125, -130), (-130, 125), (-145, 118), (118, -145), (60, -75), (-80, -20), (70, 20), (-147, 20), (20, -147)]


@pytest.mark.parametrize("T", [3, 24, 40, 65, 150])
@pytest.mark.parametrize("ex,ew", APART)
def test_scales_of_blocks_far_apart(gpu_device, T, ex, ew):
    """32-bit scales per block, as a product that is moderate of factors that are not."""
    from paper_2508_13437_amd import dmmv

    K, O = 300, 70
    for rows in (1, 128):
        x = dmmv.BlockMatrix(codes_of(T, K, T, gpu_device), powers(T, 3, ex, 1, gpu_device))
        w = dmmv.BlockMatrix(codes_of(O, K, 7, gpu_device), powers(-(-O // rows), 3, ew, 2, gpu_device), rows)
        for dtype in (torch.float32, torch.bfloat16):
            check_product(x, w, dtype)


@pytest.mark.parametrize("T", [3, 40, 150])
def test_blocks_of_many_sizes_in_a_sum(gpu_device, T):
    """A block that is large in x is small in w, another for every block; a scale of zero beside the largest."""
    from paper_2508_13437_amd import dmmv

    K, O = 1024, 70
    up = torch.tensor([[2.0 ** e for e in (120, -120, 0, 64, -90, 3, -3, 1)]], device=gpu_device)
    for x_scale, w_scale in ((up, 1.0 / up), (up, 1.5 / up)):
        x = dmmv.BlockMatrix(codes_of(T, K, T, gpu_device), x_scale.expand(T, -1))
        w = dmmv.BlockMatrix(codes_of(O, K, 7, gpu_device), w_scale.expand(O, -1))
        for dtype in (torch.float32, torch.bfloat16):
            check_product(x, w, dtype, torch.randn(O, generator=torch.Generator().manual_seed(T)).to(gpu_device))
    zero = up.clone()
    zero[0, 0] = 0.0
    x = dmmv.BlockMatrix(codes_of(T, K, T, gpu_device), zero.expand(T, -1))
    w = dmmv.BlockMatrix(codes_of(O, K, 7, gpu_device), torch.where(up > 2.0 ** 100, up, 1.0 / up).expand(O, -1))
    for dtype in (torch.float32, torch.bfloat16):
        check_product(x, w, dtype)


def matrix(rows, K, kind, exponent, seed, device, g=1):
    """kind: blocks (exponent bytes), row (32 bits, one per row, the second 0), byte row (an exponent per row)."""
    from paper_2508_13437_amd import dmmv

    nb = -(-K // 128)
    if kind == "row":
        s = powers(rows, 1, exponent, seed, device)
        if rows > 1:
            s[1] = 0.0
        s = s.expand(-1, nb)
    else:
        b = np.random.default_rng(seed).integers(127 + exponent, 129 + exponent, (-(-rows // g), nb if kind == "blocks" else 1)).astype(np.uint8)
        s = torch.from_numpy(b).to(device).expand(-1, nb)
    return dmmv.BlockMatrix(codes_of(rows, K, seed, device), s, g if kind == "blocks" else 1)


# few tokens, unaligned rows, the two sizes of the large tiles, a shared contraction, rows laid out first, a last block that is not whole
ROW_SIZES = [(3, 70, 300), (24, 70, 384), (40, 70, 300), (150, 70, 300), (200, 300, 528), (70, 600, 4112), (2304, 4600, 400), (2304, 2900, 900)]


@pytest.mark.parametrize("kx,kw,ex,ew", [("blocks", "row", 118, -118), ("blocks", "row", 118, -140), ("blocks", "row", -118, 118), ("row", "blocks", -118, 118),
                                         ("row", "blocks", 118, -118), ("row", "row", 118, -118), ("row", "row", -140, 120), ("blocks", "byte row", 118, -118),
                                         ("byte row", "blocks", -120, 118), ("byte row", "row", 118, -120)])
@pytest.mark.parametrize("T,O,K", ROW_SIZES)
def test_scales_of_rows_far_from_those_of_blocks(gpu_device, T, O, K, kx, kw, ex, ew):
    for g in (1, 128) if kw == "blocks" else (1,):
        x, w = matrix(T, K, kx, ex, T, gpu_device), matrix(O, K, kw, ew, O, gpu_device, g)
        for dtype in (torch.bfloat16, torch.float32) if T < 2000 else (torch.bfloat16,):
            check_product(x, w, dtype, torch.randn(O, generator=torch.Generator().manual_seed(T)).to(gpu_device))


def small_and_large_codes(rows, K, seed, device):
    """Codes of every size down to the smallest, 2^-9."""
    c = np.random.default_rng(seed).integers(0, 254, (rows, K)).astype(np.uint8)
    return torch.from_numpy(np.where(c & 127 == 127, 1, c).astype(np.uint8)).to(device)


@pytest.mark.parametrize("K,bx", [(1, [250]), (300, [250, 250, 250]), (300, [0, 1, 2]), (300, [4, 254, 127]), (1024, [250, 4, 0, 254, 127, 1, 246, 3])])
@pytest.mark.parametrize("T", [3, 24, 64, 65, 150])
def test_exponents_beyond_the_range_of_bf16(gpu_device, T, K, bx):
    """Bytes 0 to 254 whose products are moderate, for any number of tokens; the values of one operand alone may leave the range."""
    from paper_2508_13437_amd import dmmv

    O = 70
    b = torch.tensor([bx], dtype=torch.uint8, device=gpu_device)
    for g in (1, 128):
        for d in (0, 7):
            x = dmmv.BlockMatrix(small_and_large_codes(T, K, T, gpu_device), b.expand(T, -1))
            w = dmmv.BlockMatrix(small_and_large_codes(O, K, 7, gpu_device), (254 - b.int()).add(d).clamp(0, 254).to(torch.uint8).expand(1 if g == 128 else O, -1), g)
            for p, q in ((x, w), (dmmv.BlockMatrix(small_and_large_codes(T, K, T, gpu_device), w.scales[:1].expand(T, -1)),
                                  dmmv.BlockMatrix(small_and_large_codes(O, K, 7, gpu_device), b.expand(O, -1)))):
                for dtype in (torch.float32, torch.bfloat16):
                    check_product(p, q, dtype)


@pytest.mark.parametrize("T,O,K", ROW_SIZES)
def test_exponent_bytes_0_and_255(gpu_device, T, O, K):
    """255 is NaN, for its block's row alone, and 0 is 2^-127, in the 8-bit instructions as in 32 bits."""
    from paper_2508_13437_amd import dmmv

    nb = -(-K // 128)
    bx, bw = torch.full((T, nb), 127, dtype=torch.uint8), torch.full((O, nb), 127, dtype=torch.uint8)
    bx[0, nb - 1] = bw[3, 0] = 0
    x, w = (dmmv.BlockMatrix(codes_of(n, K, n, gpu_device), s.to(gpu_device)) for n, s in ((T, bx), (O, bw)))
    kinds = (torch.bfloat16, torch.float32) if T < 2000 else (torch.bfloat16,)
    for dtype in kinds:
        check_product(x, w, dtype)
    want = {dtype: dmmv.dmmv_block_product(x, w, dtype=dtype) for dtype in kinds}
    x.scales[T - 1, nb // 2], w.scales[O - 2, nb - 1] = 255, 255
    for dtype in kinds:
        got = dmmv.dmmv_block_product(x, w, dtype=dtype)
        assert bool(torch.isnan(got[T - 1]).all()) and bool(torch.isnan(got[:, O - 2]).all())
        rest = [o for o in range(O) if o != O - 2]
        assert torch.equal(got[:T - 1, rest], want[dtype][:T - 1, rest])


@pytest.mark.parametrize("T", [4, 40, 150])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_scales_of_a_matrix_without_columns_are_not_read(gpu_device, T, kind):
    """K = 0 by the C entry with a table of scales that holds NaN: the product is the bias."""
    from paper_2508_13437_amd import dmmv

    O = 70
    table = torch.full((256,), float("nan"), device=gpu_device) if kind == "f32" else torch.full((256,), 255, dtype=torch.uint8, device=gpu_device)
    codes = torch.zeros(256, dtype=torch.uint8, device=gpu_device)
    empty = lambda rows: dmmv._BlockMatrix(rows, 0, codes.data_ptr(), 0, table.data_ptr(), 1, 0, dmmv.DMMV_F32 if kind == "f32" else dmmv.DMMV_E8M0, 1)  # noqa: E731
    x, w = empty(T), empty(O)
    bias = torch.randn(O, generator=torch.Generator().manual_seed(T)).to(gpu_device)
    for dtype, name in ((torch.float32, dmmv.DMMV_F32), (torch.bfloat16, dmmv.DMMV_BF16)):
        y = torch.empty(T, O, dtype=dtype, device=gpu_device)
        dmmv._check(dmmv.load().dmmv_block_product(dmmv.C.addressof(x), dmmv.C.addressof(w), bias.data_ptr(), name, y.data_ptr(), O, None, 0,
                                                   torch.cuda.current_stream().cuda_stream))
        assert torch.equal(y, bias.to(dtype).expand(T, O))


@pytest.mark.parametrize("T", [3, 24, 65, 150])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_blocks_of_zeros_have_any_scale(gpu_device, T, kind):
    """Zeros of either sign with the smallest and the largest scales (what others put beside a block of zeros), in some blocks and whole rows."""
    from paper_2508_13437_amd import dmmv

    K, O = 700, 70
    nb = -(-K // 128)
    for small in (True, False):
        pair = []
        for rows, seed in ((T, 1), (O, 2)):
            codes = codes_of(rows, K, seed, gpu_device).view(torch.uint8)
            scales = torch.full((rows, nb), 127, dtype=torch.uint8, device=gpu_device) if kind == "e8m0" else powers(rows, nb, 0, seed, gpu_device)
            zero = torch.zeros(rows, nb, dtype=torch.bool)
            zero[:, 2], zero[rows // 2], zero[rows - 1, nb - 1] = True, True, True
            zero = zero.to(gpu_device)
            spread = zero.repeat_interleave(128, 1)[:, :K]
            codes[spread] = torch.where(torch.arange(int(spread.sum()), device=gpu_device) % 2 == 0, 0x00, 0x80).to(torch.uint8)
            scales[zero] = (0 if small else 254) if kind == "e8m0" else (2.0 ** -149 if small else 2.0 ** 127)
            pair.append(dmmv.BlockMatrix(codes, scales))
        for dtype in (torch.float32, torch.bfloat16):
            check_product(*pair, dtype)
