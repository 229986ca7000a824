"""The product with an activation and a residual in its epilogue against 64 bits.  Codes are integers and scales powers of two, so that
sums are exact and what is left to check is what follows them."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import layer_plain as plain
from tests import residual_plain as rp
from tests.test_gpu_block_product import block, f64, half_ulp, vals

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# few tokens (one to four rows of tiles, shares of blocks, odd ends); the general tiles; 128 x 128 tiles; shares of the contraction; rows laid out first;
# 256 x 256 tiles with exponents per block and along rows
SIZES = [(1, 1, 1), (1, 300, 1000), (1, 4096, 4096), (17, 65, 384), (24, 130, 520), (64, 129, 130), (65, 100, 96), (66, 127, 129), (129, 257, 385), (300, 513, 521),
         (128, 128, 1024), (257, 1030, 1296), (65, 1025, 3856), (200, 513, 8208), (1100, 2000, 8209), (2304, 4600, 400)]
KINDS = [("e8m0", "e8m0"), ("e8m0", "row"), ("f32", "f32")]


def operands(T, O, K, kx, kw, device, g=None):
    """Integer codes; u comes out around 3, exactly, bias included."""
    x, w = block(T, K, kx, T + O, device, integers=True), block(O, K, kw, K + O, device, integers=True, g=g)
    k = round(np.log2(np.sqrt(K) * 8))
    s = w.scales
    if s.dtype == torch.uint8:
        s.sub_(k)
    else:
        (s[:, :1] if s.stride(1) == 0 else s).mul_(2.0 ** -k)
    bias = torch.randint(-8, 9, (O,), generator=torch.Generator().manual_seed(K)).float().to(device) * 2.0 ** -k
    want = torch.from_numpy(vals(x)).to(device) @ torch.from_numpy(vals(w)).to(device).t() + bias.double()
    return x, w, bias, want.cpu().numpy()


def act_error(u, a, kind, short):
    """Of the activation of an exact u.  In 32 bits the logistic's argument has at most six roundings, its exponential two and what follows four;
    erfc is within 16 units in the last place (32 U), its argument two roundings, of which a relative t^2 + t times two
    becomes its own error, and two products.  For bf16 results a relative 2^-14."""
    tiny = np.abs(u) * 2.0 ** -118
    if kind is None or kind == "relu":
        return 0.0 * u
    if short:
        return 2.0 ** -14 * np.abs(a) + tiny
    if kind == "gelu":
        return (2 * (u * u + 2 * np.abs(u)) + 40) * U * np.abs(a) + tiny
    x = np.abs(u) if kind == "silu" else np.abs(2.0 * rp.K * (u + 0.044715 * u ** 3))
    return (6 * np.minimum(x, 200.0) + 10) * U * np.abs(a) + tiny


def check_q(q, want, e):
    """Values within a rounding of want +- e, scales between those of |want| - e and |want| + e."""
    T, O = want.shape
    got = plain.values(q.codes.cpu().numpy(), q.scales.cpu().numpy())
    scales = plain.scale_values(q.scales.cpu().numpy())
    step = plain.spread(scales, T, O, 1) * 2.0 ** -10
    assert (np.abs(got - want) <= e + np.maximum(2.0 ** -4 * (np.abs(want) + e), step)).all()
    nb = -(-O // 128)

    def scale_of(v):
        pad = np.zeros((T, nb * 128))
        pad[:, :O] = np.maximum(v, 0.0)
        a = pad.reshape(T, nb, 128).max(2)
        m, ex = np.frexp(a)                                              # a = m 2^ex, 448 = 0.875 * 2^9
        return np.where(a > 0, 2.0 ** np.maximum(ex - 9.0 + (m > 0.875), -126.0), 0.0), a > 0

    (least, there), (most, some) = scale_of(np.abs(want) - e), scale_of(np.abs(want) + e)
    # (a block whose numbers are all within e of 0 may have become zeros, and their scale is 1: GELU of -20 is 5e-88)
    assert (scales >= least)[there].all() and ((scales <= most) | (~there & (scales == 1.0)))[some].all()


def check(r, want_u, kind, residual, dtype, short):
    a = rp.act(want_u, kind)
    want = a if residual is None else a + f64(residual)
    e = act_error(want_u, a, kind, short) * 1.01 + (U * np.abs(want) if residual is not None else 0.0)
    if r.u is not None:
        assert torch.equal(r.u, torch.from_numpy(want_u).to(r.u.device).to(dtype))
    if r.y is not None:
        assert (np.abs(f64(r.y) - want) <= e + half_ulp(dtype) * 1.01 * (np.abs(want) + e)).all()
    if r.q is not None:
        check_q(r.q, want, e)


@pytest.mark.parametrize("kx,kw", KINDS)
@pytest.mark.parametrize("T,O,K", SIZES)
def test_linear(gpu_device, T, O, K, kx, kw):
    from paper_2508_13437_amd import dmmv

    for g in (1, 128) if kw == "e8m0" else (None,):
        x, w, bias, want = operands(T, O, K, kx, kw, gpu_device, g)
        gen = torch.Generator().manual_seed(T * O)
        for i, kind in enumerate((None, *rp.ACTS)):
            for dtype in (torch.float32, torch.bfloat16):
                res = torch.randn(T, O + 3, generator=gen).to(dtype).to(gpu_device)[:, 3:] if i % 2 == 0 else None
                r = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=True, q=True, u=True)
                check(r, want, kind, res, dtype, dtype == torch.bfloat16)
                if dtype == torch.float32:                       # 8 bits are made of the 32-bit numbers
                    q = dmmv.dmmv_block_quantize(r.y)
                    assert torch.equal(q.codes, r.q.codes) and torch.equal(q.scales, r.q.scales)
                again = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=True, q=True, u=True)
                assert torch.equal(again.y, r.y) and torch.equal(again.u, r.u) and torch.equal(again.q.codes, r.q.codes) and torch.equal(again.q.scales, r.q.scales)
                # one output at a time: with 8 bits the same numbers, without them those of the kernels of a plain result
                only = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=False, q=True)
                assert only.y is None and only.u is None and torch.equal(only.q.codes, r.q.codes) and torch.equal(only.q.scales, r.q.scales)
                only = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype)
                assert only.q is None and only.u is None
                check(only, want, kind, res, dtype, dtype == torch.bfloat16)
                only = dmmv.dmmv_block_linear(x, w, bias, kind, res, dtype, y=False, u=True)
                assert only.y is None and torch.equal(only.u, r.u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,O,K", [(1, 300, 1000), (64, 513, 512), (66, 130, 400), (300, 1030, 1296), (70, 300, 4096)])
def test_without_anything_it_is_the_product(gpu_device, T, O, K, dtype):
    """Any codes and scales: u and y are the product's bits (its sums have tests of their own)."""
    from paper_2508_13437_amd import dmmv

    for kx, kw in KINDS:
        x, w = block(T, K, kx, T, gpu_device), block(O, K, kw, O, gpu_device, g=128 if kw == "e8m0" else None)
        bias = torch.randn(O, device=gpu_device)
        want = dmmv.dmmv_block_product(x, w, bias, dtype)
        r = dmmv.dmmv_block_linear(x, w, bias, dtype=dtype, u=True)
        assert torch.equal(r.y, want) and torch.equal(r.u, want)


def test_eight_bits_of_few_tokens_come_from_sums_in_32_bits(gpu_device):
    """Random codes: all numbers but those that 1e-6 of the sum of magnitudes moves over a border of the grid are the quantised exact ones."""
    from paper_2508_13437_amd import dmmv

    for T in (1, 20, 64):
        x, w = block(T, 4096, "e8m0", T, gpu_device), block(512, 4096, "e8m0", 9, gpu_device, g=128)
        q = dmmv.dmmv_block_linear(x, w, y=False, q=True).q
        X, W = vals(x), vals(w)
        want = X @ W.T
        codes, scales = plain.quantize(want)
        got = q.codes.cpu().numpy()
        # a sum in 32 bits is off by some 1e-7 of sum |x w|, which is some 40 sums here: 4e-6 of steps of 2^-4: one number in some 10^4
        assert (got != codes).mean() <= 1e-3 and (q.scales.cpu().numpy() != scales).mean() <= 0.02


@pytest.mark.parametrize("T", [1, 20, 64])
def test_eight_bits_of_few_tokens_with_exponents_at_both_ends(gpu_device, T):
    """Exponents that bf16 does not hold exactly, in some blocks and rows: sums are exact still, and so are codes and scales."""
    from paper_2508_13437_amd import dmmv

    O, K = 200, 1100
    x, w = block(T, K, "e8m0", T, gpu_device, integers=True), block(O, K, "e8m0", 9, gpu_device, integers=True, g=128)
    gen = torch.Generator().manual_seed(T)
    low = torch.rand(1, x.scales.shape[1], generator=gen).to(gpu_device) < 0.4          # 2^-126 and 2^-125 against 2^123 and 2^122
    for far in (low, torch.ones_like(low)):
        xs, ws = x.scales.int(), w.scales.int()
        xs, ws = torch.where(far, xs - 125, xs), torch.where(far, ws + 125 - 3, ws - 3)
        a, b = dmmv.BlockMatrix(x.codes, xs.to(torch.uint8)), dmmv.BlockMatrix(w.codes, ws.to(torch.uint8), 128)
        want = vals(a) @ vals(b).T
        q = dmmv.dmmv_block_linear(a, b, y=False, q=True).q
        codes, scales = plain.quantize(want)
        got = q.codes.cpu().numpy()
        assert np.array_equal(np.where(got & 127, got, 0), np.where(codes & 127, codes, 0)) and np.array_equal(q.scales.cpu().numpy(), scales)
    ws = w.scales.clone()
    ws[0, 0] = 255                                                                          # NaN: the first 128 outputs
    q = dmmv.dmmv_block_linear(x, dmmv.BlockMatrix(w.codes, ws, 128), y=False, q=True).q
    assert bool((q.codes[:, :128] & 127 == 127).all()) and bool((q.codes[:, 128:] & 127 != 127).all())


def test_what_is_not_finite_stays_in_its_row(gpu_device):
    from paper_2508_13437_amd import dmmv

    for T, O, K in ((3, 300, 300), (150, 300, 300), (300, 384, 1024), (70, 300, 4096)):
        x, w, bias, want = operands(T, O, K, "e8m0", "e8m0", gpu_device, 128)
        clean = [dmmv.dmmv_block_linear(x, w, bias, kind, q=True, u=True) for kind in rp.ACTS]
        x.codes.view(torch.uint8)[T - 1, K - 1] = 0x7F
        res = torch.zeros(T, O, dtype=torch.bfloat16, device=gpu_device)
        res[0, 5], res[1, 6], res[1, 7] = float("inf"), float("-inf"), float("nan")
        for kind, c in zip(rp.ACTS, clean):
            r = dmmv.dmmv_block_linear(x, w, bias, kind, q=True, u=True)
            assert r.y[T - 1].isnan().all() and r.u[T - 1].isnan().all() and bool((r.q.codes[T - 1] & 127 == 127).all())
            assert torch.equal(r.y[:T - 1], c.y[:T - 1]) and torch.equal(r.q.codes[:T - 1], c.q.codes[:T - 1]) and torch.equal(r.u[:T - 1], c.u[:T - 1])
            r = dmmv.dmmv_block_linear(x, w, bias, kind, res, q=True)
            assert float(r.y[0, 5]) == float("inf") and float(r.y[1, 6]) == float("-inf") and r.y[1, 7].isnan()
            assert bool((r.q.codes[[0, 1, 1], [5, 6, 7]] & 127 == 127).all()) and r.y[:2].isfinite().sum() == 2 * O - 3
            # the block's other numbers keep a scale of their own
            assert bool((r.q.scales[:2] == c.q.scales[:2]).float().mean() > 0.5) and bool((r.q.scales < 255).all())


def test_activations_at_both_ends(gpu_device):
    """u from -3e38 to 3e38 and infinities through the bias: limits, no NaN."""
    from paper_2508_13437_amd import dmmv

    ends = torch.tensor([0.0, -0.0, 1e-30, -1e-30, -5.0, -13.2, -13.4, -20.0, -87.0, -90.0, -104.0, -1e4, -1e20, -3e38, float("-inf"), 5.0, 13.5, 90.0, 1e4, 1e20, 3e38,
                         float("inf"), float("nan")], device=gpu_device)
    O = len(ends)
    for T in (1, 70, 300):
        x = dmmv.BlockMatrix(torch.zeros(T, 256, dtype=torch.uint8, device=gpu_device))
        w = dmmv.BlockMatrix(torch.zeros(O, 256, dtype=torch.uint8, device=gpu_device))
        for dtype in (torch.float32, torch.bfloat16):
            for kind in rp.ACTS:
                y = f64(dmmv.dmmv_block_linear(x, w, ends, kind, dtype=dtype).y)
                u = f64(ends)
                assert np.isnan(y[:, -1]).all() and (y[:, -2] == np.inf).all() and (np.abs(y[:, 14]) <= 1e-36).all()
                fin = np.isfinite(u)
                with np.errstate(over="ignore", invalid="ignore"):
                    want = rp.act(u[fin], kind)
                want = np.where(np.isfinite(want), want, np.where(u[fin] > 0, u[fin], 0.0))
                e = act_error(np.clip(u[fin], -1e4, 1e4), np.where(np.abs(u[fin]) > 1e4, 0.0, want), kind, dtype == torch.bfloat16) + 1e-35
                lim = np.minimum(np.abs(want), 3.4e38)
                assert (np.abs(np.clip(y[:, fin], -3.4e38, 3.4e38) - want) <= e + half_ulp(dtype) * 1.01 * lim).all(), (kind, dtype)


@pytest.mark.parametrize("T,O,K", [(3, 140, 256), (66, 140, 200), (300, 300, 1024), (70, 140, 4096), (0, 5, 7), (5, 0, 7), (5, 9, 0)])
def test_rows_with_gaps_and_empty_ones(gpu_device, T, O, K):
    """Through the C entry: rows wider than the results; what lies between them stays as it was."""
    from paper_2508_13437_amd import dmmv

    lib = dmmv.load()
    for code, dtype in ((dmmv.DMMV_F32, torch.float32), (dmmv.DMMV_BF16, torch.bfloat16)):
        if K:
            x, w, bias, _ = operands(max(T, 1), max(O, 1), K, "e8m0", "e8m0", gpu_device, 128)
            x, w = (dmmv.BlockMatrix(b.codes[:n], b.scales[:-(-n // b.scale_rows)], b.scale_rows) for b, n in ((x, T), (w, O)))
            bias = bias[:O].contiguous()
        else:
            x, w = (dmmv.BlockMatrix(torch.empty(n, 0, dtype=torch.uint8, device=gpu_device)) for n in (T, O))
            bias = torch.arange(O, device=gpu_device, dtype=torch.float32)
        res = torch.randn(T, O, device=gpu_device).to(dtype)
        want = dmmv.dmmv_block_linear(x, w, bias, "silu", res, dtype, q=True, u=True)
        if K == 0:
            assert torch.equal(want.u, bias.to(dtype).expand(T, -1))
        wide = [torch.full((T + 1, O + 5), 7.0, dtype=dtype, device=gpu_device) for _ in range(2)]
        codes = torch.full((T + 1, O + 3), 77, dtype=torch.uint8, device=gpu_device)
        nb = -(-O // 128)
        scales = torch.full((T + 1, nb + 2), 66, dtype=torch.uint8, device=gpu_device)
        rw = torch.full((T, O + 1), 9.0, dtype=dtype, device=gpu_device)
        rw[:, :O] = res
        q = dmmv._BlockMatrix(T, O, codes.data_ptr(), O + 3, scales.data_ptr(), nb + 2, 1, dmmv.DMMV_E8M0, 1)
        n = lib.dmmv_block_linear_workspace_for(x._p, w._p, code, 1)
        ws = torch.empty(n + 1, dtype=torch.uint8, device=gpu_device)
        s = lib.dmmv_block_linear(x._p, w._p, bias.data_ptr() or None, 4, rw.data_ptr() or None, O + 1, code, wide[0].data_ptr(), O + 5, C.addressof(q), wide[1].data_ptr(),
                                  O + 5, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
        assert s == 0, lib.dmmv_last_error()
        for got, one in ((wide[0], want.y), (wide[1], want.u), (codes, want.q.codes), (scales, want.q.scales)):
            assert torch.equal(got[:T, :one.shape[1]], one)
            v = got.view(torch.uint8) if got.dtype == torch.uint8 else got.float()
            rest = v.clone()
            rest[:T, :one.shape[1]] = v[T, -1]
            assert bool((rest == v[T, -1]).all())


@pytest.mark.parametrize("T,O,K", [(3, 300, 256), (66, 300, 200), (300, 400, 1024), (70, 300, 4096)])
def test_scales_of_32_bits_and_blocks_first(gpu_device, T, O, K):
    """Through the C entry: the scales of the 8-bit result as floats, stored block by block."""
    from paper_2508_13437_amd import dmmv

    lib, nb = dmmv.load(), -(-O // 128)
    x, w, bias, _ = operands(T, O, K, "e8m0", "e8m0", gpu_device, 128)
    want = dmmv.dmmv_block_linear(x, w, bias, "gelu", y=False, q=True).q
    codes = torch.empty(T, O, dtype=torch.uint8, device=gpu_device)
    scales = torch.empty(nb, T + 3, dtype=torch.float32, device=gpu_device)
    q = dmmv._BlockMatrix(T, O, codes.data_ptr(), O, scales.data_ptr(), 1, T + 3, dmmv.DMMV_F32, 1)
    n = lib.dmmv_block_linear_workspace_for(x._p, w._p, dmmv.DMMV_BF16, 1)
    ws = torch.empty(n + 1, dtype=torch.uint8, device=gpu_device)
    assert lib.dmmv_block_linear(x._p, w._p, bias.data_ptr(), 2, None, 0, dmmv.DMMV_BF16, None, 0, C.addressof(q), None, 0, ws.data_ptr(), n,
                                 torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(codes, want.codes) and np.array_equal(scales[:, :T].t().cpu().numpy(), plain.scale_values(want.scales.cpu().numpy()))


def test_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    x, w, bias, _ = operands(4, 6, 200, "e8m0", "e8m0", gpu_device, 128)
    res = torch.zeros(4, 6, dtype=torch.bfloat16, device=gpu_device)
    for kw, status in ((dict(act="tanh"), -4), (dict(residual=res.float()), -3), (dict(residual=res[:3]), -2), (dict(residual=res[:, :5]), -2),
                       (dict(residual=res.cpu()), -6), (dict(bias=bias[:5]), -2), (dict(bias=bias.double()), -3), (dict(dtype=torch.float16), -3),
                       (dict(residual=res[0]), -2)):
        with pytest.raises(dmmv.DmmvError) as e:
            dmmv.dmmv_block_linear(x, w, **kw)
        assert e.value.status == status, kw
    with pytest.raises(dmmv.DmmvError) as e:
        dmmv.dmmv_block_linear(x, block(6, 201, "e8m0", 1, gpu_device))
    assert e.value.status == -2
