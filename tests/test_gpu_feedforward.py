"""The gated feed-forward block over 4-bit weights, the operators as a decoder calls them.

Against 64 bits on the block's own (unpacked) weights: what differs is the rounding of the two
8-bit inputs and of the 16-bit gate|up.  E4M3 rounds by up to 2^-4 of a value, 2.6 % in the root mean
square; it enters through x (in the gate and in the up), and through h: sqrt(3) 2.6 % = 4.5 % of
the output's norm.  8 % is allowed."""
import pytest
import torch

import decoder_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    torch_cuda()
    from paper_2109_03513_amd import feedforward
    return feedforward


def weights(esb, w4, N, K, group):
    q, alpha = esb.esb_w4_unpack(w4, N, K, group)
    return ref.dequantize(q.cpu().double(), alpha.cpu().double(), group)


@pytest.mark.parametrize("tokens", [1, 5, 48, 300])
@pytest.mark.parametrize("d,n,group,dtype", [(256, 640, 128, torch.bfloat16), (200, 333, 32, torch.float16)])
def test_block(ff, tokens, d, n, group, dtype):
    esb = ff.esb
    log("feed-forward tokens=%d d=%d ff=%d group=%d" % (tokens, d, n, group))
    w = ff.synthetic(d, n, seed=d, dtype=dtype)
    block = ff.GatedFeedForward(*w, group=group)
    g = torch.Generator().manual_seed(tokens)
    x, r = [torch.randn(tokens, d, generator=g).to(dtype) for _ in range(2)]
    y, z = block(x.cuda(), r.cuda())
    assert y.dtype == z.dtype == dtype and y.shape == z.shape == (tokens, d)
    rz, rn = ref.rmsnorm(x, w[3].cpu(), block.eps, r)
    ref.check_float(z, rz, 2.0 ** -24)
    gu = rn @ weights(esb, block.gate_up, 2 * n, d, group).t()
    want = ref.swiglu(gu[:, :n], gu[:, n:]) @ weights(esb, block.down, d, n, group).t()
    assert float((y.cpu().double() - want).norm()) <= 0.08 * float(want.norm())
    # and the weights are those that were given, within 4 bits: a group's largest weight is 6 steps
    # of 1 (2 above 4), so an error is at most a sixth of it, and 11 % in the root mean square
    back = weights(esb, block.down, d, n, group)
    given = w[2].cpu().double()
    assert float((back - given).norm()) <= 0.15 * float(given.norm())


@pytest.mark.parametrize("tokens", [1, 33])
def test_graph_replays(ff, tokens):
    block = ff.GatedFeedForward(*ff.synthetic(256, 512, seed=1))
    g = torch.Generator().manual_seed(9)
    inputs = [torch.randn(2, tokens, 256, generator=g).to(torch.bfloat16).cuda() for _ in range(4)]
    want = [block(v[0], v[1]) for v in inputs]
    x = inputs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z = block(x[0], x[1])
    for v, (ey, ez) in zip(inputs, want):
        x.copy_(v)
        graph.replay()
        assert torch.equal(y, ey) and torch.equal(z, ez)
        torch.cuda.synchronize()
        again = block(v[0], v[1])
        assert torch.equal(again[0], ey) and torch.equal(again[1], ez)


def test_refusals(ff):
    w = ff.synthetic(64, 96, seed=2)
    with pytest.raises(ValueError):
        ff.GatedFeedForward(w[0], w[1][:90], w[2])
    with pytest.raises(ValueError):
        ff.GatedFeedForward(w[0], w[1], w[0])
    block = ff.GatedFeedForward(*w, group=32)
    with pytest.raises(ValueError):
        block(torch.zeros(2, 60, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        block(torch.zeros(2, 64, dtype=torch.float64, device="cuda"))
