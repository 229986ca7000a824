"""What a call of the gradients needs by its arguments: the size function reads no array, so any aligned addresses do."""
import ctypes as C
import os
import random

import pytest

P = 4096            # an address that nothing reads


@pytest.fixture(scope="module")
def mod():
    from paper_2508_13437_amd import dmmv
    if not os.path.exists(dmmv.LIB_PATH):
        from paper_2508_13437_amd import build
        build.build(force=True)
    return dmmv


def needs(mod, T, O, K, dtype=None, x="e8m0", w="e8m0", dx=True, dw=True, dy=P, lddy=None, ld=None, codes=P):
    def matrix(rows, kind):
        nb = -(-K // 128)
        e8m0 = kind == "e8m0"
        return mod._BlockMatrix(rows, K, codes, K if ld is None else ld, None if kind == "none" else P, 1 if kind == "row" else nb, 0 if kind == "row" else 1,
                                mod.DMMV_E8M0 if e8m0 else mod.DMMV_F32, 1)
    a, b = matrix(T, x), matrix(O, w)
    return mod.load().dmmv_block_backward_workspace_for(mod.DMMV_BF16 if dtype is None else dtype, T, O, K, dy, O if lddy is None else lddy, C.addressof(a) if dw else None,
                                                        C.addressof(b) if dx else None, P if dx else None, P if dw else None)


def up(n, to):
    return -(-n // to) * to


def test_a_large_aligned_call_needs_its_bias_alone(mod):
    for T, O, K in ((4096, 11008, 4096), (16384, 28672, 8192), (4096, 4096, 4096)):
        assert 0 < needs(mod, T, O, K) <= 2.2e6
        assert needs(mod, T, O, K, x="none", w="none") == needs(mod, T, O, K) == needs(mod, T, O, K, dw=False) == needs(mod, T, O, K, dx=False, dw=False)


def test_what_is_laid_out_is_counted(mod):
    T, O, K = 4096, 11008, 4096
    parts = 2 * T * O
    assert needs(mod, T, O, K, mod.DMMV_F32) == 3 * parts                                     # three bf16 of dy
    assert needs(mod, T, O, K, w="row") == 2 * parts and needs(mod, T, O, K, w="row", dx=False) <= 2.2e6     # dx through a scale per row: two
    assert needs(mod, T, O, K, x="row", dx=False) == 3 * parts                               # dw is of 32 bits: three
    assert needs(mod, T, O, K, dy=P + 2) == parts                                             # one, with aligned rows
    assert needs(mod, T, O, K, ld=K + 1) == parts + max(T, O) * K                             # and the codes of w (those of x are fewer)
    assert needs(mod, T, O, K, codes=P + 1, dx=False) == parts + T * K
    small = mod.load().dmmv_block_backward_workspace_bytes
    assert small(T, O, K) >= 3 * parts
    # 32 bits of middle size: dy in parts; bf16 of the same: only shares of the contraction
    assert needs(mod, 777, 1365, 1003, mod.DMMV_F32) >= 3 * 2 * up(777, 128) * up(1365, 128)
    assert needs(mod, 777, 1365, 1003) <= 256 * 64 * 64 * 4 + 2.2e6


def test_never_more_than_for_any_call_of_the_sizes(mod):
    rng = random.Random(7)
    size = lambda hi: int(2 ** rng.uniform(0, hi))  # noqa: E731
    for _ in range(3000):
        T, O, K = size(14), size(14), size(13)
        if rng.random() < 0.5:
            T, O, K = up(T, 128), up(O, 128), up(K, 128)
        n = needs(mod, T, O, K, rng.choice([mod.DMMV_F32, mod.DMMV_BF16]), rng.choice(["e8m0", "row", "f32", "none"]), rng.choice(["e8m0", "row", "f32", "none"]),
                  rng.random() < 0.8, rng.random() < 0.8, P + 4 * rng.randrange(3), O + rng.randrange(3), K + rng.randrange(3), P + rng.randrange(2))
        assert n <= mod.load().dmmv_block_backward_workspace_bytes(T, O, K), (T, O, K)


def test_refused_calls_need_nothing(mod):
    assert needs(mod, 64, 64, 64, 7) == 0 and needs(mod, -1, 64, 64) == 0 and needs(mod, 64, 64, 64, lddy=63) == 0 and needs(mod, 64, 64, 64, dy=P + 1) == 0
    lib = mod.load()
    assert lib.dmmv_block_backward_workspace_for(mod.DMMV_F32, 8, 6, 300, P, 6, None, None, P, None) == 0 and lib.dmmv_last_error()
    # dx and dw only say what is asked for
    assert needs(mod, 8, 6, 300) > 0


def test_a_norm_of_nothing_needs_nothing(mod):
    lib = mod.load()
    for sizes in ((0, 0), (0, 300), (8, 0), (-1, 300), (8, -1), (8, 1 << 31)):
        assert lib.dmmv_layernorm_workspace_bytes(*sizes) == 0
    assert lib.dmmv_layernorm_workspace_bytes(8, 300) > 0
