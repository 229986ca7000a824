"""A residual block's operators together: the example's two blocks against automatic differentiation in 64 bits, captured and replayed, and one token."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def through(x, q):
    """The 8-bit values in the forward pass, x in the backward pass."""
    from paper_2508_13437_amd import dmmv

    return x + (dmmv.dmmv_block_dequantize(q, torch.float32).double() - x).detach()


def smooth(u, act):
    if act == "gelu":
        return 0.5 * u * torch.special.erfc(-u * 0.5 ** 0.5)
    if act == "relu":
        return u.clamp(min=0.0)
    return u * torch.sigmoid(u if act == "silu" else 2.0 * (2.0 / torch.pi) ** 0.5 * (u + 0.044715 * u ** 3))


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
@pytest.mark.parametrize("tokens,features,hidden", [(70, 208, 300), (1, 128, 256), (257, 130, 515)])
def test_gradients_of_the_blocks(gpu_device, tokens, features, hidden, act):
    """In 32 bits.  Every one of some twenty operators on the way sums at most 515 numbers in 32 bits, 515 * 2^-24 = 3e-5 of their magnitudes at most and
    some 1e-6 as a rule; quantised activations are the ones that the library has made."""
    import quantised_block as ex
    from paper_2508_13437_amd import dmmv

    g = torch.Generator().manual_seed(tokens)
    p = ex.parameters(features, hidden, g, gpu_device)
    blocks = ex.Blocks(p, act, torch.float32)
    h = ex.hidden_states(tokens, features, g).float().to(gpu_device)
    y = blocks.forward(h)
    dy = torch.randn(tokens, features, generator=g).to(gpu_device)
    got, dh = blocks.backward(dy)

    _, n, a, f, s, b = blocks.kept
    leaf = {k: (dmmv.dmmv_block_dequantize(blocks.w[k], torch.float32) if k in ex.WEIGHTS else v).double().requires_grad_() for k, v in p.items()}
    x = h.double().requires_grad_()
    rms = lambda v: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-5)  # noqa: E731
    t = (x - x.mean(1, keepdim=True)) * torch.rsqrt(x.var(1, correction=0, keepdim=True) + 1e-5) * leaf["gamma"] + leaf["beta"]
    t = smooth(through(t, n.q) @ leaf["w1"].t() + leaf["b1"], act)
    stream = ex.ALPHA * x + leaf["gate"] * rms(through(t, a.q) @ leaf["w2"].t() + leaf["b2"]) * leaf["post_gamma"]
    t = smooth(through(rms(stream) * leaf["pre_gamma"], s.q) @ leaf["w3"].t() + leaf["b3"], act)
    want = through(t, b.q) @ leaf["w4"].t() + leaf["b4"] + stream
    near = lambda a, b: float((a.double() - b).norm()) <= 3e-4 * float(b.norm())  # noqa: E731
    assert near(y, want.detach())
    want.backward(dy.double())
    assert near(dh, x.grad)
    for k, v in leaf.items():
        assert near(got[k], v.grad), k


def test_a_step_in_a_graph(gpu_device):
    """Forward, backward and clipping captured once, replayed on new numbers with the same eager work between the replays; two graphs at once."""
    import quantised_block as ex
    from paper_2508_13437_amd import dmmv

    g = torch.Generator().manual_seed(3)
    blocks = ex.Blocks(ex.parameters(192, 400, g, gpu_device))
    h, dy = ex.hidden_states(150, 192, g).to(gpu_device), (1e-2 * torch.randn(150, 192, generator=g)).to(torch.bfloat16).to(gpu_device)

    def step():
        y = blocks.forward(h)
        grads, dh = blocks.backward(dy)
        norm = dmmv.dmmv_gradient_clip(list(grads.values()), 0.1)
        return (y, dh, norm, *grads.values())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(step())
    for seed in range(4):
        new = torch.Generator().manual_seed(10 + seed)
        h.copy_(ex.hidden_states(150, 192, new).to(gpu_device))
        dy.copy_((10.0 ** -seed * torch.randn(150, 192, generator=new)).to(torch.bfloat16).to(gpu_device))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in out] for out in outs]
        want = step()
        torch.cuda.synchronize()
        for other in got:
            assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_two_streams_at_once(gpu_device):
    """The same step on two streams, neither waiting for the other: workspaces and results are a call's own."""
    import quantised_block as ex

    g = torch.Generator().manual_seed(4)
    blocks = [ex.Blocks(ex.parameters(256, 512, g, gpu_device)) for _ in range(2)]
    h = [ex.hidden_states(300, 256, g).to(gpu_device) for _ in range(2)]
    want = []
    for b, x in zip(blocks, h):
        y = b.forward(x)
        want.append((y, b.backward(y)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                y = blocks[i].forward(h[i])
                got[i] = (y, blocks[i].backward(y))
        torch.cuda.synchronize()
        for (y, (grads, dh)), (y0, (grads0, dh0)) in zip(got, want):
            assert torch.equal(y, y0) and torch.equal(dh, dh0) and all(torch.equal(grads[k], grads0[k]) for k in grads)


def test_the_example_runs_and_a_token_alone_is_a_row_of_the_batch(gpu_device):
    import quantised_block as ex

    r = ex.run(tokens=200, features=192, hidden=320, steps=6)
    assert all(v == v and v < float("inf") for v in r["losses"] + r["norms"])
    one, row = r["token"][0].float(), r["batch"][0].float()
    # the batch is summed by the 8-bit instructions, a token in 8 bits by others: some numbers are rounded to another neighbour on the way, each
    # by 2^-3 of itself at most, one in some hundred of 320 and fewer
    assert float((one - row).norm()) <= 0.02 * float(row.norm())
