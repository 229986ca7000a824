"""Clipping of tensors with gaps: every number that no tensor covers stays as it was."""
import pytest
import torch

from tests.test_gpu_gradient_clip import BF16, F32, check

pytestmark = pytest.mark.gpu


def views(m, c, s, o):
    return [m[:, :9], m[:, 9:8500], m[3:60, 8600:8601], m[:, 8700:8712], c.permute(0, 2, 3, 1), s[::3], o[1:], o[:1]]


def buffers(dtype, device):
    g = torch.Generator().manual_seed(3)
    return [torch.randn(n, generator=g).to(dtype).to(device) for n in ((70, 9001), (3, 5, 7, 11), (3000,), (20001,))]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_no_tensor_covers_stays(gpu_device, dtype):
    from paper_2508_13437_amd import dmmv

    whole = buffers(dtype, gpu_device)
    before, covered = [t.clone() for t in whole], [torch.zeros(t.shape, dtype=torch.bool, device=gpu_device) for t in whole]
    for v in views(*covered):
        assert not bool(v.any())                                           # the views are apart
        v.fill_(True)
    assert [int((~t).sum()) for t in covered] == [70 * (9001 - 8500 - 12) - 57, 0, 2000, 0]
    was = [v.clone() for v in views(*whole)]
    n = dmmv.dmmv_gradient_clip(views(*whole), 0.5)
    check(was, views(*whole), n, 0.5, 1e-6)
    for t, b, c in zip(whole, before, covered):
        assert torch.equal(t[~c], b[~c]) and bool((t[c] != b[c]).any())
    # and into the same places of other buffers, which are 7 elsewhere; what is read stays too
    whole, out = [t.clone() for t in before], [torch.full_like(t, 7.0) for t in before]
    assert torch.equal(dmmv.dmmv_gradient_clip(views(*whole), 0.5, out=views(*out)), n)
    check(was, views(*out), n, 0.5, 1e-6)
    for t, b, o, c in zip(whole, before, out, covered):
        assert torch.equal(t, b) and bool((o[~c] == 7.0).all())


@pytest.mark.parametrize("rows,cols,gap", [(70000, 1, 2), (3000, 7, 1), (300, 512, 1), (300, 513, 3), (5, 9000, 11)])
def test_columns_between_others(gpu_device, rows, cols, gap):
    """One tensor of a matrix, columns on both sides of it left alone, the last row's among them."""
    from paper_2508_13437_amd import dmmv

    for dtype in (F32, BF16):
        whole = torch.randn(rows, cols + 2 * gap, generator=torch.Generator().manual_seed(cols)).to(dtype).to(gpu_device)
        before = whole.clone()
        n = dmmv.dmmv_gradient_clip([whole[:, gap:gap + cols]], 0.3)
        check([before[:, gap:gap + cols]], [whole[:, gap:gap + cols]], n, 0.3, 1e-6)
        assert torch.equal(whole[:, :gap], before[:, :gap]) and torch.equal(whole[:, gap + cols:], before[:, gap + cols:])
