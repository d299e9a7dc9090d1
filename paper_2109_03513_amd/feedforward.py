"""A decoder's gated feed-forward block over 4-bit weights, from libesb's operators:

    z = x + residual                              esb_rmsnorm (the sum, and the norm in 8 bits)
    g | u = norm(z) W_gate|up^T                   esb_w4_gemm, 8-bit rows
    h = g / (1 + exp(-g)) * u                     esb_swiglu, in 8 bits
    y = h W_down^T                                esb_w4_gemm, 8-bit rows

Weights are quantized once (esb_w4_quantize: ESB(4,1) codes and a bf16 scale per group, found by
the aligner's search over candidate scales); the block returns (y, z), which the next block takes
as its x and residual.  Every call enqueues four kernels or a few more and allocates its outputs
from torch, so it can be captured into a HIP graph.

    python -m paper_2109_03513_amd.feedforward [hidden] [feed-forward]   times tokens and prompts
"""
import torch

from . import esb

CANDIDATES = 16


class GatedFeedForward:
    def __init__(self, w_gate, w_up, w_down, norm_weight=None, eps=1e-5, group=128):
        """w_gate, w_up: ff x d, w_down: d x ff (fp32, bf16 or fp16, on the device);
        norm_weight: d fp32, or None."""
        self.ff, self.d = w_gate.shape
        if w_up.shape != w_gate.shape or tuple(w_down.shape) != (self.d, self.ff):
            raise ValueError("w_gate and w_up must be ff x d, w_down d x ff")
        self.eps, self.group, self.norm_weight = eps, group, norm_weight
        factors = 1 - torch.arange(CANDIDATES, dtype=torch.float32, device=w_gate.device) / 32
        self.gate_up = esb.esb_w4_quantize(torch.cat([w_gate, w_up]), group, factors)
        self.down = esb.esb_w4_quantize(w_down, group, factors)

    def __call__(self, x, residual=None):
        """x, residual: tokens x d (bf16 or fp16); returns (y, z) in x's type."""
        z, _, x8, scale = esb.esb_rmsnorm(x, self.norm_weight, self.eps, residual=residual,
                                          want_sum=True)
        gu = esb.esb_w4_gemm(x8, self.gate_up, 2 * self.ff, self.group, x_scale=scale,
                             y_dtype=x.dtype)
        _, h8, scale = esb.esb_swiglu(gu[:, :self.ff], gu[:, self.ff:])
        y = esb.esb_w4_gemm(h8, self.down, self.d, self.group, x_scale=scale, y_dtype=x.dtype)
        return y, z


def synthetic(d, ff, seed=0, dtype=torch.bfloat16, device="cuda"):
    """Random weights of a block: (w_gate, w_up, w_down, norm_weight)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=device)

    return ((normal(ff, d) / d ** 0.5).to(dtype), (normal(ff, d) / d ** 0.5).to(dtype),
            (normal(d, ff) / ff ** 0.5).to(dtype), 1 + 0.1 * normal(d))


def _time(call, passes):
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        call()
    start.record()
    for _ in range(passes):
        call()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / passes * 1e3


def main(d=4096, ff=9216):
    block = GatedFeedForward(*synthetic(d, ff))
    for tokens in (1, 16, 64, 512, 4096):
        x = torch.randn(tokens, d, device="cuda").to(torch.bfloat16)
        r = torch.randn(tokens, d, device="cuda").to(torch.bfloat16)
        eager = _time(lambda: block(x, r), 20)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block(x, r)
        replay = _time(graph.replay, 20)
        print("%5d tokens: %8.1f us a call, %8.1f us as a graph, %7.1f TFLOP/s"
              % (tokens, eager, replay, 6.0 * tokens * d * ff / replay / 1e6), flush=True)


if __name__ == "__main__":
    import sys
    main(*[int(a) for a in sys.argv[1:3]])
