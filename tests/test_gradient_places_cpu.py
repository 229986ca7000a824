"""Where the clipped gradients may go: answered on the host, before any launch."""
import ctypes as C

from tests.test_residual_cpu import P, gradients, mod  # noqa: F401


def clip(mod, g, out=None):  # noqa: F811
    """-5: the places are taken, and the missing workspace is refused after them; -2: they are not."""
    a, b = gradients(mod, *g), None if out is None else gradients(mod, *out)
    return mod.load().dmmv_gradient_clip(len(g), C.addressof(a), None if b is None else C.addressof(b), 1.0, 0.0, None, None, None, 0, None)


def test_what_is_written_lies_in_no_other_gradient(mod):  # noqa: F811
    """A workgroup would overwrite numbers that another has yet to read."""
    f, h = mod.DMMV_F32, mod.DMMV_BF16
    a, b = (P, 1, 100, 100, f), (P + 400, 1, 100, 100, f)
    to, other = (1 << 20, 1, 100, 100, f), (1 << 21, 1, 100, 100, f)
    assert clip(mod, [a, b], [to, other]) == -5 and clip(mod, [a, b], [other, to]) == -5
    assert clip(mod, [a, b], [a, b]) == -5 and clip(mod, [a, b], [a, to]) == -5 and clip(mod, [a, b], [to, b]) == -5
    assert clip(mod, [a, b], [b, a]) == -2 and b"gradients 0 and 1" in mod.load().dmmv_last_error()       # swapped
    assert clip(mod, [a, b], [b, to]) == -2 and clip(mod, [a, b], [to, a]) == -2
    assert clip(mod, [a], [(P + 4, 1, 100, 100, f)]) == -2 and clip(mod, [(P + 4, 1, 100, 100, f)], [a]) == -2       # shifted by a number
    assert clip(mod, [a], [(P, 1, 100, 100, h)]) == -2 and clip(mod, [(P, 1, 100, 100, h)], [a]) == -2               # another type in the same place
    assert clip(mod, [a], [(P + 400, 1, 100, 100, f)]) == -5 and clip(mod, [b], [a]) == -5                            # side by side
    # columns of one matrix: read and written ones apart, by one column not, and rows of another stride
    left, right = (P, 50, 10, 24, f), (P + 40, 50, 10, 24, f)
    assert clip(mod, [left], [right]) == -5 and clip(mod, [right], [left]) == -5 and clip(mod, [left, right], [left, right]) == -5
    assert clip(mod, [left], [(P + 36, 50, 10, 24, f)]) == -2 and clip(mod, [left], [(P, 50, 10, 25, f)]) == -2
    assert clip(mod, [left, right], [right, left]) == -2
    # one row has no stride; nothing has no place
    assert clip(mod, [(P, 1, 10, 24, f)], [(P, 1, 10, 99, f)]) == -5 and clip(mod, [(P, 0, 10, 24, f), a], [(P, 0, 10, 24, f), to]) == -5


def test_gradients_that_are_only_read_may_be_the_same(mod):  # noqa: F811
    f = mod.DMMV_F32
    n = 20000
    same, to = [(P, 1, 100, 100, f)] * n, [((1 << 20) + 400 * i, 1, 100, 100, f) for i in range(n)]
    assert clip(mod, same, to) == -5
    # many tensors, each in its own place or in that of the next
    here = to + [((1 << 24) + 4 * i, 8, 1, 5000, f) for i in range(5000)]
    assert clip(mod, here, here) == -5 and clip(mod, to, to[1:] + to[:1]) == -2


def test_a_norm_is_no_number_of_the_gradients(mod):  # noqa: F811
    f, h = mod.DMMV_F32, mod.DMMV_BF16
    a, to = (P, 5, 10, 24, f), (1 << 20, 5, 10, 24, f)

    def refused(g, out=None, given=None, norm=None):
        g, out = gradients(mod, g), None if out is None else gradients(mod, out)
        status = mod.load().dmmv_gradient_clip(1, C.addressof(g), None if out is None else C.addressof(out), 1.0, 0.0, given, norm, 1 << 22, 1 << 10, None)
        return status == -2 and b"is a number of gradient 0" in mod.load().dmmv_last_error()

    for at in (P, P + 36, P + 96, P + 4 * 96 + 36):
        assert refused(a, norm=at) and refused(a, given=at) and refused(a, to, norm=at) and refused(to, a, norm=at) and refused(to, a, given=at), at
    assert refused((P + 2, 1, 9, 9, h), norm=P) and refused((P + 2, 1, 9, 9, h), norm=P + 16)


def test_a_tensor_without_gaps_may_have_any_number_of_rows(mod):  # noqa: F811
    """Rows are counted in 31 bits; where there are no gaps they need not be counted."""
    import torch

    n = (1 << 31) + 3
    for t, place in ((torch.empty(n, 2, device="meta"), (1, 2 * n, 2 * n)), (torch.empty(2, n, device="meta").t(), (2, n, n)),
                     (torch.empty(n, device="meta"), (1, n, n)), (torch.empty(n - 4, 2, device="meta"), (n - 4, 2, 2)),
                     (torch.empty(n, 3, device="meta")[:, :2], (n, 2, 3))):
        assert mod._place(t)[0] == place, t.shape


def test_what_lies_in_the_gaps_of_a_matrix(mod):  # noqa: F811
    """Columns of the same matrix are told apart number by number; anything else whose extent meets the matrix's is refused, as the header says, and the
    message does not claim more than that."""
    f, h = mod.DMMV_F32, mod.DMMV_BF16
    m = (P, 10, 20, 64, f)
    assert clip(mod, [m, (P + 80, 10, 44, 64, f)]) == -5 and clip(mod, [m, (P + 80 + 256, 3, 44, 64, f)]) == -5
    assert clip(mod, [m, (P + 80, 10, 45, 64, f)]) == -2
    for other in ((P + 80 + 256, 1, 44, 64, f), (P + 80, 3, 44, 128, f), (P + 80, 10, 88, 128, h)):
        assert clip(mod, [m, other]) == -2 and b"gradients 0 and 1 may share memory: their extents meet" in mod.load().dmmv_last_error(), other
        assert clip(mod, [m, other], [(1 << 20, 10, 20, 64, f), (1 << 21, *other[1:])]) == -5             # where they are only read
    # beside the matrix, after its last number
    assert clip(mod, [m, (P + 4 * (9 * 64 + 20), 1, 44, 64, f)]) == -5
