"""A decoder's attention block over 4-bit weights and a 4-bit cache, from libesb's operators:

    z = x + residual                              esb_rmsnorm (the sum, and the norm in 8 bits)
    q | k | v = norm(z) W_qkv^T                   esb_w4_gemm, 8-bit rows
  one token or a few of each sequence (step):
    q, k normed and rotated, k and v kept         esb_kv4_append
    o = softmax(q k^T / sqrt(d)) v                esb_kv4_attention, from the cache
  whole prompts (prompt):
    q, k normed and rotated, k and v kept         esb_kv4_append
    k normed and rotated                          esb_rope
    o from k and v themselves                     esb_attention
    y = o W_out^T                                 esb_w4_gemm

The block returns (y, z), which the next block takes as its x and residual.  The caller keeps the pages:
slots (tokens, int64) say where a call's keys and values go, pages (sequences x columns, int32) and
lengths (sequences, int32; the new tokens among them) what a sequence has there.  Every call allocates
its outputs from torch, so it can be captured into a HIP graph.

    python -m paper_2109_03513_amd.attention [hidden] [heads] [key heads]   times tokens and prompts
"""
import torch

from . import esb
from .feedforward import CANDIDATES, _time

D_EPS = 1e-6                       # of the norms over heads


def rotation_table(rows, rot, base=10000.0, device="cuda"):
    """Cosines, then sines, of every position's angles (computed in 64 bits)."""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([torch.cos(a), torch.sin(a)], 1).float()


class CachedAttention:
    def __init__(self, w_qkv, w_out, heads, kv_heads, table, pages, page=64, norm_weight=None, q_norm=None,
                 k_norm=None, eps=1e-5, group=128):
        """w_qkv: (heads + 2 kv_heads) d x hidden, rows of q, then k, then v; w_out: hidden x heads d (fp32,
        bf16 or fp16, on the device); table: as rotation_table makes it; pages, page: size of the cache;
        norm_weight: hidden fp32, or None; q_norm, k_norm: d fp32, or None for no norm over heads."""
        rows, self.hidden = w_qkv.shape
        self.d = rows // (heads + 2 * kv_heads)
        if rows != self.d * (heads + 2 * kv_heads) or tuple(w_out.shape) != (self.hidden, heads * self.d):
            raise ValueError("w_qkv must be (heads + 2 kv_heads) d x hidden, w_out hidden x heads d")
        if (q_norm is None) != (k_norm is None):
            raise ValueError("queries and keys are normed together")
        self.heads, self.kv_heads, self.page, self.table = heads, kv_heads, page, table
        self.eps, self.group, self.norm_weight = eps, group, norm_weight
        self.norms = dict(q_w=q_norm, k_w=k_norm, eps=0.0 if q_norm is None else D_EPS)
        size = esb.esb_kv4_page_size(page, kv_heads, self.d)
        if size == 0:
            raise ValueError("the cache does not take these heads or pages")
        self.cache = torch.zeros(pages, size, dtype=torch.uint8, device=w_qkv.device)
        factors = 1 - torch.arange(CANDIDATES, dtype=torch.float32, device=w_qkv.device) / 32
        self.qkv = esb.esb_w4_quantize(w_qkv, group, factors)
        self.out = esb.esb_w4_quantize(w_out, group, factors)

    def _heads(self, x, residual):
        z, _, x8, scale = esb.esb_rmsnorm(x, self.norm_weight, self.eps, residual=residual, want_sum=True)
        n = self.heads + 2 * self.kv_heads
        y = esb.esb_w4_gemm(x8, self.qkv, n * self.d, self.group, x_scale=scale, y_dtype=x.dtype)
        y = y.view(x.shape[0], n, self.d)
        return z, y[:, :self.heads], y[:, self.heads:-self.kv_heads], y[:, -self.kv_heads:]

    def _product(self, o):
        return esb.esb_w4_gemm(o.flatten(1), self.out, self.hidden, self.group)

    def step(self, x, residual, slots, positions, pages, lengths, starts=None):
        """x, residual: tokens x hidden (bf16 or fp16); starts: sequences + 1 int32, or None for one token
        of each.  Returns (y, z) in x's type."""
        z, q, k, v = self._heads(x, residual)
        q = esb.esb_kv4_append(self.cache, self.page, k, v, slots, self.table, positions, q=q, **self.norms)
        o = esb.esb_kv4_attention(q, self.cache, self.page, self.kv_heads, pages, lengths, starts=starts)
        return self._product(o), z

    def prompt(self, x, residual, slots, positions, starts):
        """Whole prompts, packed; starts: sequences + 1 int32.  Returns (y, z)."""
        z, q, k, v = self._heads(x, residual)
        # the cache takes k as it is, as in a step: rounded heads would get other codes
        q = esb.esb_kv4_append(self.cache, self.page, k, v, slots, self.table, positions, q=q, **self.norms)
        k = esb.esb_rope(None, k, self.table, positions, k_w=self.norms["k_w"], eps=self.norms["eps"])[1]
        o = esb.esb_attention(q, k, v, starts)
        return self._product(o), z


def synthetic(hidden, heads, kv_heads, d, seed=0, dtype=torch.bfloat16, device="cuda"):
    """Random weights of a block: (w_qkv, w_out)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=device)

    rows = (heads + 2 * kv_heads) * d
    return (normal(rows, hidden) / hidden ** 0.5).to(dtype), (normal(hidden, heads * d) / (heads * d) ** 0.5).to(dtype)


def main(hidden=4096, heads=32, kv_heads=8):
    d, page, seqs, longest = hidden // heads, 64, 64, 8192
    ones = torch.ones(d, device="cuda")
    columns = longest // page
    block = CachedAttention(*synthetic(hidden, heads, kv_heads, d), heads, kv_heads, rotation_table(longest, d),
                            seqs * columns, page, q_norm=ones, k_norm=ones)
    pages = torch.arange(seqs * columns, dtype=torch.int32, device="cuda").view(seqs, columns)
    for n in (1, 16, 64):
        for kept in (512, longest):
            x, r = [torch.randn(n, hidden, device="cuda").to(torch.bfloat16) for _ in range(2)]
            lengths = torch.full((n,), kept, dtype=torch.int32, device="cuda")
            slots = pages[:n, (kept - 1) // page].long() * page + (kept - 1) % page
            args = (x, r, slots, lengths - 1, pages[:n], lengths)
            eager = _time(lambda: block.step(*args), 20)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                block.step(*args)
            print("%3d tokens after %5d: %8.1f us a call, %8.1f us as a graph"
                  % (n, kept - 1, eager, _time(graph.replay, 20)), flush=True)
    for n in (512, longest):
        x, r = [torch.randn(n, hidden, device="cuda").to(torch.bfloat16) for _ in range(2)]
        at = torch.arange(n, device="cuda")
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        print("prompt of %5d: %8.1f us a call" % (n, _time(lambda: block.prompt(x, r, at, at.int(), starts), 10)),
              flush=True)


if __name__ == "__main__":
    import sys
    main(*[int(a) for a in sys.argv[1:4]])
