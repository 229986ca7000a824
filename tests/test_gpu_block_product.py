"""Product of 8-bit matrices and its gradients against 64 bits; with small integers, bit for bit."""
import numpy as np
import pytest
import torch

from tests import layer_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 1, 1), (1, 5, 127), (1, 300, 1000), (1, 4096, 4096), (2, 70, 128), (5, 129, 129), (16, 64, 256), (17, 65, 384), (31, 200, 640), (64, 256, 512), (65, 100, 96),
         (128, 128, 1024), (129, 257, 385), (200, 70, 96), (300, 513, 520), (257, 1030, 1300), (512, 768, 2048), (7, 3, 20000), (1300, 40, 272)]


def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U      # 8 and 24 significant bits


def f64(t):
    return t.double().cpu().numpy()


def block(rows, cols, kind, seed, device, integers=False, pad=0, g=None):
    """kind: e8m0, f32 (a scale per block), row (32 bits, one per row), none."""
    from paper_2508_13437_amd import dmmv

    r = np.random.default_rng(seed)
    if integers:                                              # magnitudes at most 8: sums of 4096 products with scales stay exact
        v = r.integers(-8, 9, (rows, cols + pad)).astype(np.float32)
    else:
        v = r.standard_t(4.0, (rows, cols + pad)).astype(np.float32) * 20.0
    codes = torch.from_numpy(np.clip(v, -448, 448)).to(device).to(torch.float8_e4m3fn)[:, pad:]
    g = g or (1 if kind != "f32" or seed % 2 else 128)
    shape = (-(-rows // g), -(-cols // 128))
    if kind == "none":
        return dmmv.BlockMatrix(codes)
    if kind == "e8m0":
        b = r.integers(126, 128, shape) if integers else r.integers(110, 130, shape)
        s = torch.from_numpy(b.astype(np.uint8))
    elif kind == "row":
        g, s = 1, torch.from_numpy((2.0 ** r.integers(-1, 2, (rows, 1)) if integers else r.uniform(0.01, 3.0, (rows, 1))).astype(np.float32))
        s = s.to(device).expand(-1, shape[1])
    else:
        s = torch.from_numpy((2.0 ** r.integers(-1, 2, shape) if integers else r.uniform(0.01, 3.0, shape)).astype(np.float32))
    return dmmv.BlockMatrix(codes, s.to(device), g)


def vals(q):
    return plain.values(q.codes.view(torch.uint8).cpu().numpy(), None if q.scales is None else q.scales.cpu().numpy(), q.scale_rows)


KINDS = [("e8m0", "e8m0"), ("e8m0", "row"), ("f32", "f32"), ("e8m0", "f32"), ("none", "row"), ("row", "none")]


@pytest.mark.parametrize("kx,kw", KINDS)
@pytest.mark.parametrize("T,O,K", SIZES)
def test_product(gpu_device, T, O, K, kx, kw):
    from paper_2508_13437_amd import dmmv

    seed = 3 * T + 5 * O + 7 * K
    for dtype, pad in ((torch.float32, 0), (torch.bfloat16, 1)):
        x = block(T, K, kx, seed, gpu_device, pad=pad)
        w = block(O, K, kw, seed + 1, gpu_device, pad=5 * pad, g=128 if kw == "e8m0" else None)
        bias = torch.randn(O, generator=torch.Generator().manual_seed(seed)).to(gpu_device)
        X, W = vals(x), vals(w)
        want, size = X @ W.T + f64(bias), np.abs(X) @ np.abs(W).T + np.abs(f64(bias))
        got = dmmv.dmmv_block_product(x, w, bias, dtype=dtype)
        # a sum of K exact products, three roundings for scales; bf16: what the 8-bit instructions drop, 13 bits below the
        # largest product of a step (2^-11 of the sum of all at most, with codes drawn like these or more unevenly)
        e = (K + 8) * 2 * U * size + (2.0 ** -10 * size if dtype == torch.bfloat16 else 0.0)
        assert (np.abs(f64(got) - want) <= e + half_ulp(dtype) * 1.01 * (np.abs(want) + e)).all()
        assert np.linalg.norm(f64(got) - want) <= (2e-6 + 1.01 * half_ulp(dtype)) * np.linalg.norm(want) + 1e-6 * np.linalg.norm(size) / np.sqrt(K)
        assert torch.equal(got, dmmv.dmmv_block_product(x, w, bias, dtype=dtype))


# the large tiles, many steps and more blocks than a table of exponents holds, with and without aligned rows; small and large
# tiles of the general kernel
LARGE = [(1300, 2100, 8512), (2304, 4600, 400), (1100, 2000, 8209), (70, 2500, 16640), (900, 1800, 1072)]


@pytest.mark.parametrize("kx,kw", [("e8m0", "e8m0"), ("e8m0", "row"), ("f32", "f32")])
@pytest.mark.parametrize("T,O,K", LARGE)
def test_large_products_of_integers_are_exact(gpu_device, T, O, K, kx, kw):
    from paper_2508_13437_amd import dmmv

    for g in (1, 128) if kw == "e8m0" else (None,):
        x = block(T, K, kx, T + O, gpu_device, integers=True)
        w = block(O, K, kw, K + O, gpu_device, integers=True, g=g)
        want = torch.from_numpy(vals(x)).to(gpu_device) @ torch.from_numpy(vals(w)).to(gpu_device).t()
        bias = torch.arange(O, device=gpu_device, dtype=torch.float32) - 7.0
        assert torch.equal(dmmv.dmmv_block_product(x, w, bias, dtype=torch.float32).double(), want + bias)
        # integers beyond 2^13 times the smallest product are what the 8-bit instructions drop: none here
        assert torch.equal(dmmv.dmmv_block_product(x, w, bias, dtype=torch.bfloat16), (want + bias).to(torch.bfloat16))


# few tiles and a long contraction, which workgroups share: a last share that is shorter, a last block that is not whole, more blocks
# in a share than a table of exponents holds, rows laid out first; few tokens by tiles
@pytest.mark.parametrize("kx,kw", [k for k in KINDS if "f32" not in k])
@pytest.mark.parametrize("T,O,K", [(33, 100, 4112), (65, 1025, 3856), (200, 513, 8208), (40, 128, 80000), (120, 3000, 17001), (24, 11008, 3600)])
def test_shared_contractions(gpu_device, T, O, K, kx, kw):
    from paper_2508_13437_amd import dmmv

    for g in (1, 128) if kw == "e8m0" else (None,):
        x, w = block(T, K, kx, T + O, gpu_device), block(O, K, kw, K + O, gpu_device, g=g)
        X, W = (torch.from_numpy(vals(q)).to(gpu_device) for q in (x, w))
        bias = torch.randn(O, device=gpu_device)
        for b in (bias, None):
            got = dmmv.dmmv_block_product(x, w, b)
            want, size = X @ W.t(), X.abs() @ W.abs().t()
            if b is not None:
                want, size = want + b.double(), size + b.double().abs()
            e = (K + 8) * 2 * U * size + 2.0 ** -10 * size                       # as in test_product
            assert bool(((got.double() - want).abs() <= e + half_ulp(torch.bfloat16) * 1.01 * (want.abs() + e)).all())
            assert float((got.double() - want).norm()) <= (2e-6 + 1.01 * half_ulp(torch.bfloat16)) * float(want.norm()) + 1e-6 * float(size.norm()) / K ** 0.5
            assert torch.equal(got, dmmv.dmmv_block_product(x, w, b))
        if K > 40000:                                                            # (scales and codes that a sum in 32 bits holds exactly)
            continue
        x, w = block(T, K, kx, T + O, gpu_device, integers=True), block(O, K, kw, K + O, gpu_device, integers=True, g=g)
        want = torch.from_numpy(vals(x)).to(gpu_device) @ torch.from_numpy(vals(w)).to(gpu_device).t()
        assert torch.equal(dmmv.dmmv_block_product(x, w), want.to(torch.bfloat16))
        x.codes.view(torch.uint8)[T - 1, K - 1] = 0x7F
        got = dmmv.dmmv_block_product(x, w)
        assert torch.isnan(got[T - 1]).all() and torch.equal(got[:T - 1], want[:T - 1].to(torch.bfloat16))


@pytest.mark.parametrize("kx,kw", KINDS)
@pytest.mark.parametrize("T,O,K", [s for s in SIZES if s[2] <= 4096])
def test_product_of_integers_is_exact(gpu_device, T, O, K, kx, kw):
    from paper_2508_13437_amd import dmmv

    x = block(T, K, kx, T + O, gpu_device, integers=True)
    w = block(O, K, kw, K + O, gpu_device, integers=True, g=128 if kw == "e8m0" else None)
    got = dmmv.dmmv_block_product(x, w, dtype=torch.float32)
    assert np.array_equal(f64(got), vals(x) @ vals(w).T)


def test_product_of_what_is_not_finite(gpu_device):
    from paper_2508_13437_amd import dmmv

    for T in (3, 150):
        x, w = block(T, 300, "e8m0", 1, gpu_device, integers=True), block(140, 300, "e8m0", 2, gpu_device, integers=True)
        want = vals(x) @ vals(w).T
        x.codes.view(torch.uint8)[1, 200] = 0x7F
        w.codes.view(torch.uint8)[130, 299] = 0xFF
        w.scales[7, 1] = 255
        got = f64(dmmv.dmmv_block_product(x, w, dtype=torch.float32))
        nan = np.zeros((T, 140), bool)
        nan[1], nan[:, 130], nan[:, 7] = True, True, True
        assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("K", [256, 200])
@pytest.mark.parametrize("T", [3, 40, 150])
def test_zeros_times_large_scales(gpu_device, T, K):
    """The scales' product is beyond the range, the rows and columns of zeros are not."""
    from paper_2508_13437_amd import dmmv

    g = torch.Generator().manual_seed(K)
    codes = lambda rows: torch.randint(0x30, 0x40, (rows, K), generator=g, dtype=torch.uint8).to(gpu_device)
    bias = torch.randn(80, generator=g).to(gpu_device)
    byte, number = torch.full((1, 2), 227, dtype=torch.uint8, device=gpu_device), torch.full((1, 2), 2.0 ** 100, device=gpu_device)
    x, w = codes(T), codes(80)
    x[1], w[7] = 0, 0
    for s in (byte, number):
        for rows in (s.expand(-1, 2), s[:, :1].expand(-1, 2)):
            a, b = dmmv.BlockMatrix(x, rows.expand(T, -1)), dmmv.BlockMatrix(w, rows.expand(80, -1).contiguous())
            for p, q in ((a, b), (dmmv.BlockMatrix(x, rows.expand(T, -1).contiguous()), b)):
                for dtype in (torch.float32, torch.bfloat16):
                    y = dmmv.dmmv_block_product(p, q, bias, dtype)
                    assert torch.equal(y[1], bias.to(dtype)) and torch.equal(y[:, 7], bias[7].to(dtype).expand(T))
                    assert not torch.isfinite(y[0, :7]).any()


def test_empty_products(gpu_device):
    from paper_2508_13437_amd import dmmv

    bias = torch.randn(6, device=gpu_device)
    for T, O, K in ((0, 6, 20), (4, 0, 20), (4, 6, 0)):
        y = dmmv.dmmv_block_product(block(T, K, "none", 1, gpu_device), block(O, K, "none", 1, gpu_device), bias[:O], dtype=torch.float32)
        assert y.shape == (T, O) and torch.equal(y, bias[:O].expand(T, O))
    x, w = block(4, 20, "none", 1, gpu_device), block(6, 20, "none", 1, gpu_device)
    dx, dw, db = dmmv.dmmv_block_backward(torch.empty(0, 6, device=gpu_device), block(0, 20, "none", 1, gpu_device), w)
    assert dx.shape == (0, 20) and (dw == 0).all() and (db == 0).all()
    dx, dw, db = dmmv.dmmv_block_backward(torch.empty(4, 0, device=gpu_device), x, block(0, 20, "none", 1, gpu_device))
    assert (dx == 0).all() and dw.shape == (0, 20) and db.shape == (0,)


def test_rows_far_apart(gpu_device):
    """Codes whose rows lie 2^31 bytes apart: offsets past 32 bits."""
    from paper_2508_13437_amd import dmmv

    ld = (1 << 31) + 16
    src, w = block(3, 272, "e8m0", 1, gpu_device, integers=True), block(80, 272, "e8m0", 2, gpu_device, integers=True)
    buf = torch.empty(2 * ld + 272, dtype=torch.uint8, device=gpu_device)
    codes = buf.as_strided((3, 272), (ld, 1))
    codes.copy_(src.codes.view(torch.uint8))
    far = dmmv.BlockMatrix(codes, src.scales)
    assert torch.equal(dmmv.dmmv_block_product(far, w), dmmv.dmmv_block_product(src, w))
    assert torch.equal(dmmv.dmmv_block_product(w, far), dmmv.dmmv_block_product(w, src))
    dy = torch.randn(3, 80, device=gpu_device)
    assert torch.equal(dmmv.dmmv_block_backward(dy, far, w)[1], dmmv.dmmv_block_backward(dy, src, w)[1])
    dy = torch.randn(80, 3, device=gpu_device)
    assert torch.equal(dmmv.dmmv_block_backward(dy, w, far)[0], dmmv.dmmv_block_backward(dy, w, src)[0])


def gradients(T, O, dtype, seed, device, pad=0, integers=False):
    r = np.random.default_rng(seed)
    d = r.integers(-8, 9, (T, O + pad)) if integers else r.standard_normal((T, O + pad)) * np.exp(r.standard_normal((T, 1)))
    return torch.from_numpy(d.astype(np.float32)).to(dtype).to(device)[:, pad:]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kx,kw", [("e8m0", "e8m0"), ("e8m0", "row"), ("f32", "f32"), ("row", "none")])
@pytest.mark.parametrize("T,O,K", [s for s in SIZES if s[2] <= 4096] + [(5000, 40, 70)])
def test_backward(gpu_device, T, O, K, kx, kw, dtype):
    from paper_2508_13437_amd import dmmv

    seed = T + O + K
    pad = seed % 2
    x, w = block(T, K, kx, seed, gpu_device, pad=pad), block(O, K, kw, seed + 1, gpu_device, pad=pad, g=128 if kw == "e8m0" else None)
    dy = gradients(T, O, dtype, seed, gpu_device, pad)
    X, W, D = vals(x), vals(w), f64(dy)
    got = dmmv.dmmv_block_backward(dy, x, w)
    # sums of n products of numbers of 24 bits at most: parts left out and a scale's rounding are a few units more
    for g, want, size, n, dt in ((got[0], D @ W, np.abs(D) @ np.abs(W), O, dtype), (got[1], D.T @ X, np.abs(D).T @ np.abs(X), T, torch.float32),
                                 (got[2], D.sum(0), np.abs(D).sum(0), T, torch.float32)):
        e = (n + 12) * 2 * U * size
        assert (np.abs(f64(g) - want) <= e + half_ulp(dt) * 1.01 * (np.abs(want) + e)).all()
        assert np.linalg.norm(f64(g) - want) <= (2e-6 + 1.01 * half_ulp(dt)) * np.linalg.norm(want) + 1e-6 * np.linalg.norm(size) / np.sqrt(n)
    again = dmmv.dmmv_block_backward(dy, x, w)
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    assert torch.equal(dmmv.dmmv_block_backward(dy, None, w, dw=False, dbias=False)[0], got[0])
    assert torch.equal(dmmv.dmmv_block_backward(dy, x, None, dx=False)[1], got[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,O,K", [s for s in SIZES if s[2] <= 4096])
def test_backward_of_integers_is_exact(gpu_device, T, O, K, dtype):
    from paper_2508_13437_amd import dmmv

    x = block(T, K, "e8m0", T + O, gpu_device, integers=True)
    w = block(O, K, "e8m0", K + O, gpu_device, integers=True, g=128)
    dy = gradients(T, O, dtype, T, gpu_device, integers=True)
    dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
    want = torch.from_numpy(f64(dy) @ vals(w)).to(dtype)
    assert np.array_equal(f64(dx), f64(want))
    assert np.array_equal(f64(dw), f64(dy).T @ vals(x)) and np.array_equal(f64(db), f64(dy).sum(0))


# the large tiles: whole and partial ones, contractions of whole pairs of steps, a step and a part more, less than a pair
@pytest.mark.parametrize("T,O,K", [(512, 768, 1024), (1000, 1352, 784), (328, 264, 272), (1096, 1072, 2064), (2050, 520, 400), (260, 2312, 272)])
def test_large_backward_of_integers_is_exact(gpu_device, T, O, K):
    from paper_2508_13437_amd import dmmv

    for kind, g in (("e8m0", 128), ("e8m0", 1), ("none", 1)):
        x, w = block(T, K, kind, T + O, gpu_device, integers=True, g=1), block(O, K, kind, K + O, gpu_device, integers=True, g=g)
        dy = gradients(T, O, torch.bfloat16, T, gpu_device, integers=True)
        dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
        X, W = (torch.from_numpy(vals(q)).to(gpu_device) for q in (x, w))
        assert torch.equal(dx, (dy.double() @ W).to(torch.bfloat16))
        assert torch.equal(dw.double(), dy.double().t() @ X) and torch.equal(db.double(), dy.double().sum(0))


@pytest.mark.parametrize("T,O,K", [(2048, 4096, 2064), (2050, 4101, 2051), (4099, 2049, 1999)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_gradients_laid_out_first(gpu_device, T, O, K, dtype):
    """32-bit gradients, scales per row and rows that are not aligned, at sizes that the large tiles take."""
    from paper_2508_13437_amd import dmmv

    for kx, kw in (("e8m0", "e8m0"), ("row", "row"), ("e8m0", "row")):
        x, w = block(T, K, kx, T + O, gpu_device, integers=True, g=1), block(O, K, kw, K + O, gpu_device, integers=True, g=128 if kw == "e8m0" else None)
        dy = gradients(T, O, dtype, T, gpu_device, integers=True, pad=1 if dtype == torch.bfloat16 else 0)
        dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
        X, W = (torch.from_numpy(vals(q)).to(gpu_device) for q in (x, w))
        assert torch.equal(dx, (dy.double() @ W).to(dtype))
        assert torch.equal(dw.double(), dy.double().t() @ X) and torch.equal(db.double(), dy.double().sum(0))
    # numbers that need all their bits
    x, w = block(T, K, "e8m0", 5, gpu_device, g=1), block(O, K, "row", 6, gpu_device)
    dy = gradients(T, O, dtype, 7, gpu_device)
    dx, dw, _ = dmmv.dmmv_block_backward(dy, x, w)
    X, W = (torch.from_numpy(vals(q)).to(gpu_device) for q in (x, w))
    for g, want, size, n, dt in ((dx, dy.double() @ W, dy.double().abs() @ W.abs(), O, dtype), (dw, dy.double().t() @ X, dy.double().t().abs() @ X.abs(), T, torch.float32)):
        # (a bf16 result may come from products of 16 bits)
        e = ((n + 12) * 2 * U + (2.0 ** -15 if dt == torch.bfloat16 else 0.0)) * size
        assert bool(((g.double() - want).abs() <= e + half_ulp(dt) * 1.01 * (want.abs() + e)).all())
        assert float((g.double() - want).norm()) <= (2e-6 + 1.01 * half_ulp(dt)) * float(want.norm())


# small tiles of 32-bit gradients cut into parts beforehand: short rows, a part of a step, shares of the contraction, more tiles than
# compute units, whole steps
@pytest.mark.parametrize("T,O,K", [(64, 64, 3), (100, 70, 130), (65, 2050, 400), (2051, 66, 390), (777, 1365, 1003), (1601, 1024, 1000)])
def test_small_gradients_laid_out_first(gpu_device, T, O, K):
    from paper_2508_13437_amd import dmmv

    for kx, kw in (("e8m0", "e8m0"), ("row", "row"), ("none", "row"), ("row", "e8m0")):
        for integers in (True, False):
            x = block(T, K, kx, T + O, gpu_device, integers=integers, g=1)
            w = block(O, K, kw, K + O, gpu_device, integers=integers, g=128 if kw == "e8m0" else None)
            dy = gradients(T, O, torch.float32, T + K, gpu_device, integers=integers, pad=1)
            dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
            X, W = (torch.from_numpy(vals(q)).to(gpu_device) for q in (x, w))
            D = dy.double()
            for g, want, size, n in ((dx, D @ W, D.abs() @ W.abs(), O), (dw, D.t() @ X, D.t().abs() @ X.abs(), T), (db, D.sum(0), D.abs().sum(0), T)):
                if integers:
                    assert torch.equal(g.double(), want)
                else:
                    assert bool(((g.double() - want).abs() <= (n + 12) * 2 * U * size + U * 1.01 * want.abs()).all())
    # what is not finite stays in its rows and columns
    x, w = block(T, K, "e8m0", 5, gpu_device, g=1), block(O, K, "row", 6, gpu_device)
    w.codes.view(torch.uint8)[O - 1, 1] = 0x7F
    x.codes.view(torch.uint8)[T - 1, 2] = 0x7F
    dy = gradients(T, O, torch.float32, 7, gpu_device)
    dy[3, 5] = float("inf")
    dx, dw, db = dmmv.dmmv_block_backward(dy, x, w)
    bad = torch.zeros(T, K, dtype=torch.bool, device=gpu_device)
    bad[:, 1] = bad[3, :] = True
    assert torch.equal(~torch.isfinite(dx), bad)
    bad = torch.zeros(O, K, dtype=torch.bool, device=gpu_device)
    bad[:, 2] = bad[5, :] = True
    assert torch.equal(~torch.isfinite(dw), bad)
    assert torch.isinf(db[5]) and torch.isfinite(db).sum() == O - 1


def test_gradient_against_differences(gpu_device):
    """sum(dy * product) moves by dx (dw) times the scale when one integer code moves by one: exactly."""
    from paper_2508_13437_amd import dmmv

    x, w = block(9, 300, "e8m0", 5, gpu_device, integers=True), block(70, 300, "e8m0", 6, gpu_device, integers=True, g=128)
    dy = gradients(9, 70, torch.float32, 4, gpu_device, integers=True)
    dx, dw, _ = (f64(t) for t in dmmv.dmmv_block_backward(dy, x, w))
    at = lambda: float((f64(dmmv.dmmv_block_product(x, w, dtype=torch.float32)) * f64(dy)).sum())  # noqa: E731
    base = at()
    for q, grad, places in ((x, dx, ((0, 0), (4, 150), (8, 299))), (w, dw, ((0, 5), (33, 128), (69, 299)))):
        for i, j in places:
            old = q.codes[i, j].float()
            new = old - 1.0 if float(old) > 0 else old + 1.0
            q.codes[i, j] = new.to(torch.float8_e4m3fn)
            s = plain.spread(plain.scale_values(q.scales.cpu().numpy()), q.rows, q.cols, q.scale_rows)[i, j]
            assert at() - base == grad[i, j] * s * float(new - old)
            q.codes[i, j] = old.to(torch.float8_e4m3fn)


def test_backward_keeps_what_is_not_finite(gpu_device):
    from paper_2508_13437_amd import dmmv

    for dtype in (torch.float32, torch.bfloat16):
        x, w = block(150, 300, "e8m0", 5, gpu_device, integers=True), block(140, 300, "e8m0", 6, gpu_device, integers=True, g=128)
        dy = gradients(150, 140, dtype, 4, gpu_device, integers=True)
        want = [f64(t) for t in dmmv.dmmv_block_backward(dy, x, w)]
        dy[3, 7], dy[149, 139] = float("nan"), float("inf")
        got = [f64(t) for t in dmmv.dmmv_block_backward(dy, x, w)]
        rows, cols = np.zeros(150, bool), np.zeros(140, bool)
        rows[[3, 149]], cols[[7, 139]] = True, True
        assert not np.isfinite(got[0][rows]).any() and np.array_equal(got[0][~rows], want[0][~rows])
        assert not np.isfinite(got[1][cols]).any() and np.array_equal(got[1][~cols], want[1][~cols])
        assert not np.isfinite(got[2][cols]).any() and np.array_equal(got[2][~cols], want[2][~cols])


def test_broadcast_and_transposed_gradients(gpu_device):
    from paper_2508_13437_amd import dmmv

    x, w = block(40, 200, "e8m0", 5, gpu_device), block(70, 200, "e8m0", 6, gpu_device, g=128)
    one = torch.randn(1, 70, device=gpu_device)
    for dy in (one.expand(40, 70), torch.randn(70, 40, device=gpu_device).t(), torch.ones((), device=gpu_device).expand(40, 70)):
        for p, q in zip(dmmv.dmmv_block_backward(dy, x, w), dmmv.dmmv_block_backward(dy.contiguous(), x, w)):
            assert torch.equal(p, q)


def test_refusals(gpu_device):
    from paper_2508_13437_amd import dmmv

    x, w = block(4, 200, "e8m0", 1, gpu_device), block(6, 200, "e8m0", 2, gpu_device)
    dy = torch.randn(4, 6, device=gpu_device)
    for call, status in ((lambda: dmmv.dmmv_block_product(x, block(6, 199, "none", 1, gpu_device)), -2),
                         (lambda: dmmv.dmmv_block_product(x, w, dtype=torch.float16), -3),
                         (lambda: dmmv.dmmv_block_product(x, w, torch.ones(5, device=gpu_device)), -2),
                         (lambda: dmmv.dmmv_block_product(x, w, torch.ones(6, dtype=torch.float64, device=gpu_device)), -3),
                         (lambda: dmmv.dmmv_block_backward(dy[:3], x, w), -2), (lambda: dmmv.dmmv_block_backward(dy[:, :5], x, w), -2),
                         (lambda: dmmv.dmmv_block_backward(dy.half(), x, w), -3), (lambda: dmmv.dmmv_block_backward(dy, None, w), -1),
                         (lambda: dmmv.dmmv_block_backward(dy, x, None), -1), (lambda: dmmv.dmmv_block_backward(dy.cpu(), x, w), -6)):
        with pytest.raises(dmmv.DmmvError) as e:
            call()
        assert e.value.status == status
    lib, s = dmmv.load(), torch.cuda.current_stream().cuda_stream
    y = torch.empty(4, 6, device=gpu_device)
    assert lib.dmmv_block_product(x._p, w._p, None, dmmv.DMMV_F32, y.data_ptr(), 5, None, 0, s) == -2
    assert lib.dmmv_block_product(x._p, None, None, dmmv.DMMV_F32, y.data_ptr(), 6, None, 0, s) == -1
    assert lib.dmmv_block_product(x._p, w._p, None, dmmv.DMMV_F32, None, 6, None, 0, s) == -1
    need = lib.dmmv_block_backward_workspace_bytes(4, 6, 200)
    assert need > 0
    assert lib.dmmv_block_backward(dmmv.DMMV_F32, 4, 6, 200, dy.data_ptr(), 6, x._p, w._p, None, 0, None, 0, y.data_ptr(), None, 0, s) == -5
    assert lib.dmmv_block_product_workspace_bytes(-1, 5, 5) == 0 and lib.dmmv_block_backward_workspace_bytes(1 << 40, 5, 5) == 0
