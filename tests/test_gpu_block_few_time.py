"""Few tokens: a shorter contraction takes less time, and results do not depend on how blocks are requested."""
import pytest
import torch

from tests.test_gpu_block_linear import KINDS, operands

pytestmark = pytest.mark.gpu


def graphed(calls):
    """us a call, one after another in a graph."""
    for c in calls:
        c()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = [c() for c in calls * 6]
    times = []
    for _ in range(9):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3 / len(kept))
    return sorted(times)[len(times) // 2]


@pytest.mark.parametrize("eight", [False, True])
def test_a_quarter_of_the_weights_takes_less_time(gpu_device, eight):
    """32 tokens, 11008 outputs, contractions of 512 and 2048: 5.6 MB against 22.5 MB of weights.  Requests for blocks that are not there made both take
    nearly the same."""
    from paper_2508_13437_amd import dmmv

    g, us = torch.Generator(device=gpu_device).manual_seed(1), []
    for K in (512, 2048):
        x = dmmv.dmmv_block_quantize(torch.randn(32, K, generator=g, device=gpu_device))
        ws = [dmmv.dmmv_block_quantize(torch.randn(11008, K, generator=g, device=gpu_device), 128) for _ in range(4)]
        us.append(graphed([(lambda w=w: dmmv.dmmv_block_linear(x, w, y=False, q=True)) if eight else (lambda w=w: dmmv.dmmv_block_product(x, w)) for w in ws]))
    assert us[0] <= 0.75 * us[1], us


# blocks a wavefront around the six and five from which they go in a ring, with and without a last block that is not whole
@pytest.mark.parametrize("kx,kw", KINDS[:2])
@pytest.mark.parametrize("K", [127, 640, 2433, 2560, 3200, 3201, 3585, 5200])
def test_few_tokens_of_any_number_of_blocks(gpu_device, K, kx, kw):
    """Integer codes and powers of two: exact sums."""
    from paper_2508_13437_amd import dmmv

    for T, O in ((1, 40), (16, 300), (17, 40), (17, 8192), (17, 8208), (32, 300), (33, 40), (64, 300)):
        x, w, bias, want = operands(T, O, K, kx, kw, gpu_device, 128 if kw == "e8m0" else None)
        want = torch.from_numpy(want).to(gpu_device)
        assert torch.equal(dmmv.dmmv_block_product(x, w, bias), want.to(torch.bfloat16)) and torch.equal(dmmv.dmmv_block_product(x, w, bias, torch.float32).double(), want)
        r = dmmv.dmmv_block_linear(x, w, bias, u=True, q=True)
        assert torch.equal(r.y, want.to(torch.bfloat16)) and torch.equal(r.u, r.y)
        q = dmmv.dmmv_block_quantize(want.float())
        assert torch.equal(q.codes, r.q.codes) and torch.equal(q.scales, r.q.scales)
