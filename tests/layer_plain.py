"""The operators of include/dmmv_layer.h in 64 bits, element by element from their definitions (CPU, numpy)."""
import numpy as np

E4M3 = np.empty(256)
for _c in range(256):
    _e, _m = (_c >> 3) & 15, _c & 7
    _v = _m * 2.0 ** -9 if _e == 0 else (8 + _m) * 2.0 ** (_e - 10)
    E4M3[_c] = (-1.0 if _c & 128 else 1.0) * (np.nan if _c & 127 == 127 else _v)


def spread(scales, rows, cols, g):
    return np.repeat(np.repeat(scales, g, 0)[:rows], 128, 1)[:, :cols]


def scale_values(scales):
    if scales.dtype == np.uint8:
        return np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return scales.astype(np.float64)


def values(codes, scales, g=1):
    v = E4M3[codes]
    return v if scales is None else v * spread(scale_values(scales), *codes.shape, g)


def quantize(x, g=1):
    """codes (uint8, NaN as 0x7F) and exponent bytes of x (float64 holding float32 or bf16 values)."""
    rows, cols = x.shape
    nr, nb = -(-rows // g), -(-cols // 128)
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((nr, nb), np.uint8)
    grid = E4M3[:127]                                        # 0 .. 448 ascending
    for i in range(nr):
        for j in range(nb):
            blk = x[i * g:(i + 1) * g, j * 128:(j + 1) * 128]
            fin = np.isfinite(blk)
            a = np.abs(blk[fin]).max() if fin.any() else 0.0
            e = 0
            if a > 0:
                e = -126
                while 448.0 * 2.0 ** e < a:
                    e += 1
            scales[i, j] = e + 127
            v = np.where(fin, np.abs(blk), 0.0) / 2.0 ** e
            hi = np.clip(np.searchsorted(grid, v), 0, 126)   # first grid value >= v
            lo = np.maximum(hi - 1, 0)
            up = (grid[hi] - v < v - grid[lo]) | ((grid[hi] - v == v - grid[lo]) & (hi % 2 == 0)) | (hi == 0)
            c = np.where(up, hi, lo).astype(np.uint8)
            c = np.where(np.signbit(blk), c | 128, c)
            codes[i * g:(i + 1) * g, j * 128:(j + 1) * 128] = np.where(fin, c, 0x7F)
    return codes, scales


def norm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def norm_grad(dy, x, gamma, mean, rstd):
    h = (x - mean[:, None]) * rstd[:, None]
    a = dy * gamma
    dx = rstd[:, None] * (a - a.mean(1, keepdims=True) - h * (a * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)
