"""Clipping of more tensors than a launch takes, with more partial sums than two launches have."""
import math

import pytest
import torch

from tests.test_gpu_gradient_clip import BF16, F32, check, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count,numbers", [(200, 131072), (130, 300007), (2500, 8192), (129, 131072)])
def test_norm_and_clip(gpu_device, count, numbers):
    """2064 to 3200 parts, of 3 to 40 launches."""
    from paper_2508_13437_amd import dmmv

    for types, max_norm in (([F32, BF16], 1e-3), ([BF16], 1e6), ([F32], 0.25)):
        ts = tensors([(numbers,)] * count, types, count, gpu_device)
        before = [t.clone() for t in ts]
        out = [torch.full_like(t, 7.0) for t in ts]
        n = dmmv.dmmv_gradient_norm(ts)
        assert torch.equal(dmmv.dmmv_gradient_clip(ts, max_norm, out=out), n) and all(torch.equal(a, b) for a, b in zip(ts, before))
        check(before, out, n, max_norm, 1e-6)
        assert torch.equal(dmmv.dmmv_gradient_clip(ts, max_norm), n) and all(torch.equal(a, b) for a, b in zip(ts, out))
        given = [t.clone() for t in before]
        assert torch.equal(dmmv.dmmv_gradient_clip(given, max_norm, norm=n), n)
        check(before, given, n, max_norm, 1e-6)
    ts[-1][-1] = math.nan
    assert dmmv.dmmv_gradient_clip(ts, 1.0).isnan() and all(bool(t.isnan().all()) for t in ts)


def test_captured(gpu_device):
    from paper_2508_13437_amd import dmmv

    whole = torch.zeros(160 * 131072, device=gpu_device)
    out = torch.zeros_like(whole)
    g, o = (dmmv.Gradients(list(w.view(160, -1).unbind(0))) for w in (whole, out))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dmmv.dmmv_gradient_clip(g, 0.1, out=o)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n = dmmv.dmmv_gradient_clip(g, 0.1, out=o)
    for seed in range(4):
        whole.copy_(10.0 ** -seed * torch.randn(whole.shape, generator=torch.Generator(device=gpu_device).manual_seed(seed), device=gpu_device))
        graph.replay()
        torch.cuda.synchronize()
        norm, got = n.clone(), out.clone()
        assert torch.equal(dmmv.dmmv_gradient_clip(g, 0.1, out=o), norm) and torch.equal(out, got)
        check([whole], [got], norm, 0.1, 1e-6)


def test_time_grows_with_the_tensors_not_with_their_square(gpu_device):
    """8192 tensors, 128 launches of 1024 parts each: reading, and reading and writing in place, are three times the norm's reading and its launches
    twice.  With all parts read by every workgroup of every launch it was 13 times."""
    from paper_2508_13437_amd import dmmv

    g = dmmv.Gradients(list(torch.randn(8192, 131072, device=gpu_device).unbind(0)))

    def fastest(call):
        times = []
        for i in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call(i)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times[1:])

    norm = fastest(lambda i: dmmv.dmmv_gradient_norm(g))
    clip = fastest(lambda i: dmmv.dmmv_gradient_clip(g, 0.5 ** i))
    assert clip <= 6 * norm, (clip, norm)


def test_more_rows_than_31_bits_count(gpu_device):
    """Without gaps the rows need not be counted."""
    from paper_2508_13437_amd import dmmv

    t = torch.zeros((1 << 31) + 3, 2, dtype=BF16, device=gpu_device)
    t[0, 1], t[1 << 31, 0], t[-1, 1] = 3.0, -4.0, 12.0
    assert float(dmmv.dmmv_gradient_norm([t])) == 13.0 and float(dmmv.dmmv_gradient_clip([t], 6.5, 0.0, out=[t])) == 13.0
    assert (float(t[0, 1]), float(t[1 << 31, 0]), float(t[-1, 1])) == (1.5, -2.0, 6.0)
