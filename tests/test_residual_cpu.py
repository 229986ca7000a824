"""Refusals and sizes of a residual block's operators that need no GPU: every call here is answered before any GPU work."""
import ctypes as C
import os

import numpy as np
import pytest

from tests import residual_plain as plain

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


def test_linear_refusals(mod):
    lib, f = mod.load(), mod.DMMV_F32
    x, w, q = block(mod, 8, 300), block(mod, 6, 300), block(mod, 8, 6)

    def call(xx=x, ww=w, bias=P, act=0, res=P, ldr=6, dtype=f, y=P, ldy=6, qq=None, u=None, ldu=6, ws=P, n=1 << 20):
        at = lambda b: None if b is None else C.addressof(b)  # noqa: E731
        return lib.dmmv_block_linear(at(xx), at(ww), bias, act, res, ldr, dtype, y, ldy, at(qq), u, ldu, ws, n, None)

    for dtype in (mod.DMMV_F64, mod.DMMV_E8M0, -1, 9):
        assert call(dtype=dtype) == -3
    for act in (-1, 5, 1 << 20):
        assert call(act=act) == -4 and lib.dmmv_last_error()
    assert call(xx=None) == -1 and call(ww=None) == -1 and call(ww=block(mod, 6, 301)) == -2
    assert call(bias=P + 2) == -2 and call(ldr=5) == -2 and call(ldy=5) == -2 and call(u=P, ldu=5) == -2 and call(res=P + 1) == -2
    assert call(qq=block(mod, 8, 7)) == -2 and call(qq=block(mod, 8, 6, scale_rows=128)) == -8 and call(qq=block(mod, 8, 6, scales=None)) == -1
    need = lib.dmmv_block_linear_workspace_for(C.addressof(x), C.addressof(w), f, 1)
    assert need == 8 * 6 * 4                                          # few tokens: the 32-bit results
    assert call(qq=q, ws=None, n=0) == -5 and call(qq=q, n=need - 1) == -5 and call(qq=q, ws=P + 8) == -5
    assert call(y=None) == 0                                          # nothing is asked for


def test_linear_workspace(mod):
    lib = mod.load()

    def need(T, O, K, dtype, q, **kw):
        x, w = block(mod, T, K, **kw), block(mod, O, K, **kw)
        return lib.dmmv_block_linear_workspace_for(C.addressof(x), C.addressof(w), dtype, q)

    f32, bf16 = mod.DMMV_F32, mod.DMMV_BF16
    assert need(4096, 11008, 4096, bf16, 0) == need(4096, 11008, 4096, bf16, 1) == 0        # tiles have whole blocks
    assert need(4096, 11008, 4096, f32, 0) == 0 and need(4096, 11008, 4096, f32, 1) == 4 * 4096 * 11008
    assert need(64, 4096, 11008, bf16, 1) == 4 * 64 * 4096                                   # few tokens, never shared
    assert need(65, 4096, 11008, bf16, 0) == need(65, 4096, 11008, bf16, 1) > 0              # shares of the contraction
    assert need(500, 1777, 2731, bf16, 1) == 4 * 500 * 1777
    laid = need(4096, 11008, 4095, bf16, 0)
    assert laid == need(4096, 11008, 4095, bf16, 1) == (4096 + 11008) * 4096
    assert need(0, 5, 5, f32, 1) == 0 and need(5, 5, 5, 7, 1) == 0 and need(-1, 5, 5, f32, 1) == 0
    a, b = block(mod, 5, 5), block(mod, 5, 6)
    assert lib.dmmv_block_linear_workspace_for(C.addressof(a), C.addressof(b), f32, 1) == 0


def test_activation_refusals(mod):
    lib, f = mod.load(), mod.DMMV_F32
    need = lib.dmmv_activation_workspace_bytes(8, 300)
    assert need == 1200

    def call(dtype=f, dy=P, lddy=300, u=P, ldu=300, act=1, du=P, lddu=300, db=P, ws=P, n=need, rows=8):
        return lib.dmmv_activation_backward(dtype, rows, 300, dy, lddy, u, ldu, act, du, lddu, db, ws, n, None)

    assert call(dtype=1) == -3 and call(act=0) == -4 and call(act=5) == -4 and call(rows=-1) == -2
    assert call(dy=None) == -1 and call(u=None) == -1 and call(lddy=299) == -2 and call(ldu=299) == -2 and call(lddu=299) == -2 and call(db=P + 2) == -2
    assert call(ws=None) == -5 and call(n=need - 1) == -5
    assert call(du=None, db=None) == 0 and call(du=None, db=None, ws=None) == 0
    for sizes in ((0, 300), (8, 0), (-1, 3), (3, 1 << 31)):
        assert lib.dmmv_activation_workspace_bytes(*sizes) == 0


def norm(mod, gamma=None, beta=None, eps=1e-5, rms=0):
    return mod._Norm(gamma, beta, eps, rms)


def test_residual_norm_refusals(mod):
    lib, fl = mod.load(), mod.DMMV_F32
    ok, q = norm(mod), block(mod, 8, 300)

    def call(dtype=fl, rows=8, f=P, ldf=300, h=P, ldh=300, alpha=1.0, gate=None, ldgate=300, gate_rows=8, post=ok, pre=ok, v=P, ldv=300, y=P, ldy=300, qq=q,
             stat=P):
        at = lambda b: None if b is None else C.addressof(b)  # noqa: E731
        return lib.dmmv_residual_norm(dtype, rows, 300, f, ldf, h, ldh, alpha, gate, ldgate, gate_rows, at(post), at(pre), v, ldv, y, ldy, at(qq), stat, P, P, P, None)

    assert call(dtype=1) == -3 and call(rows=-1) == -2 and call(f=None) == -1 and call(h=None) == -1
    for alpha in (float("nan"), float("inf"), float("-inf")):
        assert call(alpha=alpha) == -4
    for bad in (norm(mod, eps=-1e-5), norm(mod, eps=float("nan")), norm(mod, eps=float("inf")), norm(mod, rms=2)):
        assert call(post=bad) == -4 and call(pre=bad) == -4
    assert call(post=norm(mod, gamma=P + 1)) == -2 and call(pre=norm(mod, beta=P + 2)) == -2
    assert call(pre=None) == -1 and call(pre=None, qq=None) == -1 and call(pre=None, y=None) == -1
    assert call(gate=P, gate_rows=0) == -2 and call(gate=P, gate_rows=-3) == -2 and call(gate=P, gate_rows=4, ldgate=299) == -2 and call(gate=P + 2) == -2
    assert call(ldf=299) == -2 and call(ldh=299) == -2 and call(ldv=299) == -2 and call(ldy=299) == -2 and call(stat=P + 1) == -2
    assert call(qq=block(mod, 7, 300)) == -2 and call(qq=block(mod, 8, 300, scale_rows=128)) == -8
    assert call(rows=0, f=None, h=None, v=None, y=None, qq=None) == 0


def test_residual_norm_backward_refusals(mod):
    lib, fl = mod.load(), mod.DMMV_F32
    ok, rms = norm(mod), norm(mod, rms=1)
    need = lib.dmmv_residual_norm_workspace_bytes(8, 300, 4)
    assert need > 0

    def call(dtype=fl, rows=8, dy=P, dv=P, f=P, v=P, alpha=1.0, gate=P, gate_rows=4, post=ok, pre=ok, pm=P, pr=P, m=P, r=P, df=P, lddf=300, dh=P, dgate=P,
             lddgate=300, dpg=P, dpb=P, dg=P, db=P, ws=P, n=need):
        at = lambda b: None if b is None else C.addressof(b)  # noqa: E731
        return lib.dmmv_residual_norm_backward(dtype, rows, 300, dy, 300, dv, 300, f, 300, v, 300, alpha, gate, 300, gate_rows, at(post), at(pre), pm, pr, m, r,
                                               df, lddf, dh, 300, dgate, lddgate, dpg, dpb, dg, db, ws, n, None)

    assert call(dtype=3) == -3 and call(rows=-1) == -2 and call(alpha=float("nan")) == -4
    assert call(dy=None) == -1 and call(pre=None) == -1 and call(dy=None, dv=None, pre=None, dg=None, db=None) == -1
    assert call(f=None) == -1 and call(v=None) == -1 and call(gate=None) == -1 and call(post=None) == -1
    assert call(pm=None) == -1 and call(pr=None) == -1 and call(m=None) == -1 and call(r=None) == -1
    assert call(post=rms, pm=None, ws=None) == -5 and call(pre=rms, m=None, ws=None) == -5          # an RMS norm has no mean
    assert call(pre=None, dy=None, dg=None) == -1 and call(pre=None, dy=None, db=None) == -1
    assert call(lddf=299) == -2 and call(lddgate=299) == -2 and call(gate_rows=0) == -2 and call(dpg=P + 1) == -2
    assert call(ws=None) == -5 and call(n=need - 1) == -5 and call(ws=P + 64) == -5
    assert call(df=None, dh=None, dgate=None, dpg=None, dpb=None, dg=None, db=None) == 0
    for sizes in ((0, 300, 1), (8, 0, 1), (-1, 300, 1), (8, 1 << 31, 1)):
        assert lib.dmmv_residual_norm_workspace_bytes(*sizes) == 0


def test_residual_norm_workspace_is_partial_sums(mod):
    """At most some 1500 workgroups' five sums (a group of its own for 1024 gates at most), and four numbers a row for long rows."""
    lib = mod.load()
    for rows in (1, 7, 513, 4096, 100000):
        for cols in (1, 300, 4096, 5000, 40000):
            for gate in (0, 1, 3, 100, rows):
                n = lib.dmmv_residual_norm_workspace_bytes(rows, cols, gate)
                assert 0 < n <= (1600 * 5 * cols) * 4 + 16 * rows + 256, (rows, cols, gate)


def test_more_than_a_launch_takes_is_refused(mod):
    """Rows times threads from 2^32 on, gradients of rows of more than 65535 x 2048 columns, bias gradients of more than 2^27: before any launch."""
    lib, dtype, rms = mod.load(), mod.DMMV_BF16, norm(mod, rms=1)
    ok = C.addressof(rms)

    def forward(rows, cols):
        return lib.dmmv_residual_norm(dtype, rows, cols, P, cols, P, cols, 1.0, None, 0, 0, ok, ok, P, cols, P, cols, None, None, P, None, P, None)

    def backward(rows, cols):
        return lib.dmmv_residual_norm_backward(dtype, rows, cols, P, cols, P, cols, P, cols, P, cols, 1.0, None, 0, 0, ok, ok, None, P, None, P, P, cols, P, cols,
                                               None, 0, None, None, None, None, P, 1 << 60, None)

    for rows, cols in ((1 << 25, 1000), (1 << 24, 2000), (1 << 23, 4096), (1 << 23, 8192), (1 << 22, 16384), (1 << 22, 40000), ((1 << 26) + 1, 512)):
        assert forward(rows, cols) == -2 and b"launch" in lib.dmmv_last_error()
    assert backward(1 << 24, 9000) == -2 and b"launch" in lib.dmmv_last_error()
    assert backward(1, 65535 * 2048 + 1) == -2 and b"launch" in lib.dmmv_last_error()
    assert lib.dmmv_activation_backward(dtype, 1, (1 << 27) + 1, P, 1 << 28, P, 1 << 28, 1, P, 1 << 28, P, P, 1 << 60, None) == -2


def gradients(mod, *g):
    a = (mod._Gradient * max(len(g), 1))()
    for i, v in enumerate(g):
        a[i] = mod._Gradient(*v)
    return a


def test_gradient_refusals(mod):
    lib, f, b = mod.load(), mod.DMMV_F32, mod.DMMV_BF16
    one = gradients(mod, (P, 4, 10, 12, f))
    need = lib.dmmv_gradient_workspace_bytes(1, C.addressof(one))
    assert need == 8                                                  # one sum of the four rows

    def norm_of(g, n=1, out=P, ws=P, size=1 << 20):
        return lib.dmmv_gradient_norm(n, None if g is None else C.addressof(g), out, ws, size, None)

    def clip(g, o=None, n=1, max_norm=1.0, eps=0.0, given=None, norm=P, ws=P, size=1 << 20):
        return lib.dmmv_gradient_clip(n, None if g is None else C.addressof(g), None if o is None else C.addressof(o), max_norm, eps, given, norm, ws, size, None)

    for bad, status in (((P, 4, 10, 12, 1), -3), ((P, -1, 10, 12, f), -2), ((P, 4, -1, 12, f), -2), ((P, 4, 10, 9, f), -2), ((None, 4, 10, 12, f), -1),
                        ((P + 2, 4, 10, 12, f), -2), ((P + 1, 4, 10, 12, b), -2), ((P, 4, 1 << 42, 1 << 42, f), -2), ((P, 1 << 31, 1, 1, f), -2)):
        g = gradients(mod, bad)
        assert norm_of(g) == status and clip(g) == status and clip(one, g) == status, bad
        assert lib.dmmv_gradient_workspace_bytes(1, C.addressof(g)) == 0
    assert norm_of(None) == -1 and norm_of(one, n=-1) == -2 and norm_of(one, out=None) == -1 and norm_of(one, out=P + 2) == -2
    assert norm_of(one, ws=None) == -5 and norm_of(one, size=need - 1) == -5 and norm_of(one, ws=P + 4) == -5
    for v in (-1.0, float("nan"), float("inf")):
        assert clip(one, max_norm=v) == -4 and clip(one, eps=v) == -4
    assert clip(one, gradients(mod, (P, 4, 11, 12, f))) == -2 and clip(one, gradients(mod, (P, 3, 10, 12, f))) == -2
    assert clip(one, given=P + 1) == -2 and clip(one, norm=P + 2) == -2 and clip(one, ws=None) == -5 and clip(one, size=need - 1) == -5


def test_gradients_that_share_memory_are_refused(mod):
    lib, f, b = mod.load(), mod.DMMV_F32, mod.DMMV_BF16

    def apart(*g):
        """Whether the check lets them pass: the workspace is refused after it."""
        a = gradients(mod, *g)
        status = lib.dmmv_gradient_clip(len(g), C.addressof(a), None, 1.0, 0.0, None, None, None, 0, None)
        assert status in (-5, -2)
        return status == -5

    assert not apart((P, 1, 10, 10, f), (P, 1, 10, 10, f)) and not apart((P, 1, 10, 10, f), (P + 36, 1, 1, 1, f))
    assert apart((P, 1, 10, 10, f), (P + 40, 1, 10, 10, f)) and apart((P + 40, 1, 10, 10, f), (P, 1, 10, 10, f))
    # columns of one matrix, in any order; one more column is one too many
    assert apart((P, 5, 4, 10, f), (P + 16, 5, 6, 10, f)) and apart((P + 16, 5, 6, 10, f), (P, 5, 4, 10, f), (P + 200, 1, 3, 3, f))
    assert not apart((P, 5, 5, 10, f), (P + 16, 5, 6, 10, f)) and not apart((P, 5, 4, 10, f), (P + 16, 5, 7, 10, f))
    assert not apart((P, 5, 4, 10, f), (P + 16, 5, 6, 11, f)) and not apart((P, 5, 4, 10, f), (P + 16, 1, 6, 10, f))
    # one that lies inside another, with a third between them in the order of addresses
    assert not apart((P, 50, 4, 10, f), (P + 16, 50, 2, 10, f), (P + 1600, 3, 4, 10, f))
    assert not apart((P, 1, 10, 10, b), (P + 18, 1, 1, 1, b)) and apart((P, 1, 10, 10, b), (P + 20, 1, 1, 1, b))
    # many pairs of halves, and more columns of one matrix than are compared
    assert apart(*[(P + 400 * i + 20 * k, 10, 5, 10, f) for i in range(20000) for k in (0, 1)])
    assert not apart(*[(P + 4 * i, 2, 1, 20000, f) for i in range(20000)]) and b"too many" in lib.dmmv_last_error()
    # empty ones have no place
    assert apart((P, 0, 10, 10, f), (P, 1, 10, 10, f), (None, 4, 0, 0, f))


def test_a_tensor_that_is_too_large_is_refused_before_any_launch(mod):
    """After more tensors than a launch takes: none of those is launched either (no workspace is given)."""
    lib, f = mod.load(), mod.DMMV_F32
    g = gradients(mod, *[(P + 64 * i, 1, 1, 1, f) for i in range(70)], (1 << 40, (1 << 31) - 1, 8193, 8200, f))
    at = C.addressof(g)
    assert lib.dmmv_gradient_workspace_bytes(71, at) == 0 and lib.dmmv_last_error()
    assert lib.dmmv_gradient_norm(71, at, P, None, 0, None) == -2 and lib.dmmv_gradient_clip(71, at, None, 1.0, 0.0, P, None, None, 0, None) == -2


def test_gradient_workspace_counts_every_launch(mod):
    lib, f = mod.load(), mod.DMMV_F32
    many = gradients(mod, *[(P, 1, 1, 1, f)] * 130)
    assert lib.dmmv_gradient_workspace_bytes(130, C.addressof(many)) == 130 * 8
    big = gradients(mod, *[(P, 1, 1 << 30, 1 << 30, f)] * 65)
    assert lib.dmmv_gradient_workspace_bytes(65, C.addressof(big)) == 2 * 1024 * 8
    assert lib.dmmv_gradient_workspace_bytes(0, None) == 0


@pytest.mark.parametrize("kind", plain.ACTS)
def test_slopes_are_the_activations_derivatives(kind):
    """The reference itself: differences of act, whose error at this step is about 1e-10."""
    u = np.concatenate([np.linspace(-6, 6, 241) + 0.013, [-20.0, 20.0]])
    d = (plain.act(u + 1e-5, kind) - plain.act(u - 1e-5, kind)) / 2e-5
    assert np.abs(d - plain.slope(u, kind)).max() < 1e-9
