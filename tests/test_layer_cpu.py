"""Refusals and sizes of the layer operators that need no GPU: every call here is answered before any GPU work."""
import ctypes as C
import os

import pytest

P = 4096            # an address that nothing reads


@pytest.fixture(scope="module")
def mod():
    from paper_2508_13437_amd import dmmv
    if not os.path.exists(dmmv.LIB_PATH):
        from paper_2508_13437_amd import build
        build.build(force=True)
    return dmmv


def block(mod, rows=8, cols=300, **other):
    q = mod._BlockMatrix(rows, cols, P, cols, P, -(-cols // 128), 1, mod.DMMV_E8M0, 1)
    for k, v in other.items():
        setattr(q, k, v)
    return q


@pytest.mark.parametrize("other,status", [
    (dict(rows=-1), -2), (dict(cols=1 << 31), -2), (dict(codes=None), -1), (dict(ld=299), -2), (dict(ld=1 << 62), -2), (dict(scales=None), -1),
    (dict(scale_type=7), -3), (dict(scale_rows=2), -2), (dict(scale_row_stride=-1), -2), (dict(scale_row_stride=2), -2),
    (dict(scale_block_stride=0), -2), (dict(scale_type=0, scales=P + 2), -2)])
def test_quantize_refuses_what_it_cannot_write(mod, other, status):
    lib = mod.load()
    q = block(mod, **other)
    if "scale_type" in other and other["scale_type"] == 0:
        q.scale_type = mod.DMMV_F32
    assert lib.dmmv_block_quantize(mod.DMMV_F32, P, 300, C.addressof(q), None) == status
    assert lib.dmmv_last_error()


def test_types_and_arrays(mod):
    lib = mod.load()
    q = block(mod)
    at = C.addressof(q)
    for dtype in (mod.DMMV_F64, mod.DMMV_E8M0, -1, 9):
        assert lib.dmmv_block_quantize(dtype, P, 300, at, None) == -3
        assert lib.dmmv_block_dequantize(at, dtype, P, 300, None) == -3
        assert lib.dmmv_block_product(at, at, None, dtype, P, 8, None, 0, None) == -3
        assert lib.dmmv_layernorm(dtype, 8, 300, P, 300, None, None, 1e-5, P, 300, None, None, None, None, None) == -3
    assert lib.dmmv_block_quantize(mod.DMMV_F32, None, 300, at, None) == -1
    assert lib.dmmv_block_quantize(mod.DMMV_F32, P + 2, 300, at, None) == -2
    assert lib.dmmv_block_quantize(mod.DMMV_BF16, P, 299, at, None) == -2
    assert lib.dmmv_block_quantize(mod.DMMV_F32, P, 300, None, None) == -1
    other = block(mod, cols=301)
    assert lib.dmmv_block_product(at, C.addressof(other), None, mod.DMMV_F32, P, 8, None, 0, None) == -2
    assert lib.dmmv_block_product(at, at, P + 1, mod.DMMV_F32, P, 8, None, 0, None) == -2


def test_norm_refusals(mod):
    lib = mod.load()
    f = mod.DMMV_F32
    for eps in (-1e-5, float("nan"), float("inf")):
        assert lib.dmmv_layernorm(f, 8, 300, P, 300, None, None, eps, P, 300, None, None, None, None, None) == -4
    q = block(mod, rows=7)
    assert lib.dmmv_layernorm(f, 8, 300, P, 300, None, None, 0.0, None, 0, C.addressof(q), None, None, None, None) == -2
    q = block(mod, scale_rows=128)
    assert lib.dmmv_layernorm(f, 8, 300, P, 300, None, None, 0.0, None, 0, None, C.addressof(q), None, None, None) == -8
    need = lib.dmmv_layernorm_workspace_bytes(8, 300)
    q = block(mod)
    both = lambda x, xq, mean, ws, n: lib.dmmv_layernorm_backward(f, 8, 300, P, 300, x, 300, xq, None, mean, P, P, 300, P, P, ws, n, None)
    assert need > 0
    assert both(P, C.addressof(q), P, P, need) == -1 and both(None, None, P, P, need) == -1 and both(P, None, None, P, need) == -1
    assert both(P, None, P, None, need) == -5 and both(P, None, P, P, need - 1) == -5 and both(P, None, P, P + 128, need) == -5


def test_backward_refusals(mod):
    lib = mod.load()
    x, w = block(mod, 8, 300), block(mod, 6, 300)
    f, need = mod.DMMV_F32, lib.dmmv_block_backward_workspace_bytes(8, 6, 300)

    def call(T=8, O=6, K=300, xx=x, ww=w, lddx=300, lddw=300, ws=P, n=None):
        return lib.dmmv_block_backward(f, T, O, K, P, 6, C.addressof(xx) if xx else None, C.addressof(ww) if ww else None, P, lddx, P, lddw, P, ws,
                                       need if n is None else n, None)

    assert need > 0
    assert call(xx=None) == -1 and call(ww=None) == -1
    assert call(xx=w) == -2 and call(ww=x) == -2 and call(K=299) == -2 and call(T=-8) == -2
    assert call(lddx=299) == -2 and call(lddw=299) == -2
    assert call(ws=None) == -5 and call(n=need - 1) == -5


def test_workspace_sizes(mod):
    lib = mod.load()
    for sizes in ((-1, 5, 5), (5, -1, 5), (5, 5, 1 << 31)):
        assert lib.dmmv_block_product_workspace_bytes(*sizes) == 0 and lib.dmmv_block_backward_workspace_bytes(*sizes) == 0
    assert lib.dmmv_layernorm_workspace_bytes(-1, 5) == 0 and lib.dmmv_layernorm_workspace_bytes(0, 0) >= 0
    assert lib.dmmv_block_product_workspace_bytes(4096, 11008, 4096) == 0              # aligned rows are read where they are
    ragged = lib.dmmv_block_product_workspace_bytes(4096, 11008, 4095)
    assert ragged == (4096 + 11008) * 4096
    # a gradient that is laid out in parts: three bf16 for every number of dy, and the codes
    assert lib.dmmv_block_backward_workspace_bytes(4096, 4096, 4096) >= 3 * 2 * 4096 * 4096
    # the same bytes serve a gradient after the other: no more than dy in parts, padded, and partial sums for every compute unit
    for T, O, K in ((1, 11008, 4096), (64, 64, 3), (777, 1365, 1003), (2051, 66, 390)):
        up = lambda n: -(-n // 128) * 128
        assert lib.dmmv_block_backward_workspace_bytes(T, O, K) <= 3 * 2 * up(T) * up(O) + max(T, O) * up(K) + 256 * 64 * 64 * 4 + 256 * O * 4 + 1024
