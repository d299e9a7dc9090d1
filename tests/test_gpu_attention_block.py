"""The attention block over 4-bit weights and a 4-bit cache, the operators as a decoder calls them.

Against 64 bits on the block's own weights, and for steps on its own cache.  What differs is the E4M3
rounding of the block's input, 2.6 % of a value in the root mean square: of v as much, and of q and k,
whose scores (of about 1) it moves by sqrt(2) 2.6 %, so of the weights that much again; together
4.5 % of the output's norm.  10 % is allowed, so that a wrong position, key or head fails."""
import pytest
import torch

import attention_ref as ref
import decoder_ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def at():
    torch_cuda()
    from paper_2109_03513_amd import attention
    return attention


def weights(esb, w4, N, K, group):
    q, alpha = esb.esb_w4_unpack(w4, N, K, group)
    return decoder_ref.dequantize(q.cpu().double(), alpha.cpu().double(), group)


class Model:
    """A block, a few sequences of its cache, and what 64 bits make of its calls."""

    def __init__(self, at, heads, kv, d, dtype, norms, hidden=256, group=64, page=16, columns=12, seqs=3):
        self.at, self.dtype, self.page, self.columns, self.seqs = at, dtype, page, columns, seqs
        g = torch.Generator().manual_seed(d)
        n = [None, None] if not norms else [1 + 0.2 * torch.randn(d, generator=g) for _ in range(2)]
        self.norms, self.tab = n, ref.table(page * columns, d)
        self.norm_weight = 1 + 0.1 * torch.randn(hidden, generator=g)
        cuda = [None if w is None else w.cuda() for w in n]
        self.b = at.CachedAttention(*at.synthetic(hidden, heads, kv, d, seed=d, dtype=dtype), heads, kv, self.tab.cuda(),
                                    seqs * columns + 3, page, norm_weight=self.norm_weight.cuda(), q_norm=cuda[0],
                                    k_norm=cuda[1], group=group)
        self.pages = torch.randperm(seqs * columns + 3, generator=g)[:seqs * columns].view(seqs, columns).int().cuda()
        self.w_qkv = weights(at.esb, self.b.qkv, (heads + 2 * kv) * d, hidden, group)
        self.w_out = weights(at.esb, self.b.out, hidden, heads * d, group)
        self.kept = [0] * seqs

    def batch(self, counts, seed):
        g = torch.Generator().manual_seed(seed)
        x, r = [torch.randn(sum(counts), self.b.hidden, generator=g).to(self.dtype) for _ in range(2)]
        pos = [torch.arange(self.kept[i], self.kept[i] + n) for i, n in enumerate(counts)]
        self.kept = [k + n for k, n in zip(self.kept, counts)]
        slots = [self.pages[i].cpu().long()[p // self.page] * self.page + p % self.page for i, p in enumerate(pos)]
        starts = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32).cuda()
        lengths = torch.tensor(self.kept, dtype=torch.int32).cuda()
        return x, r, torch.cat(slots).cuda(), torch.cat(pos).int().cuda(), starts, lengths

    def expected(self, x, r, positions, counts, cached):
        b = self.b
        z, n = decoder_ref.rmsnorm(x, self.norm_weight, b.eps, r)
        qkv = (n @ self.w_qkv.t()).reshape(x.shape[0], -1, b.d)
        eps = 0.0 if self.norms[0] is None else self.at.D_EPS
        q, _ = ref.turn(qkv[:, :b.heads], self.norms[0], eps, self.tab, positions.cpu(), False)
        k, _ = ref.turn(qkv[:, b.heads:-b.kv_heads], self.norms[1], eps, self.tab, positions.cpu(), False)
        v, o, a = qkv[:, -b.kv_heads:], [], 0
        for i, c in enumerate(counts):
            ki, vi = (k[a:a + c], v[a:a + c]) if not cached else self.read(i)
            last = torch.arange(c) + ki.shape[0] - c
            o.append(ref.attend(q[a:a + c], ki, vi, last, b.d ** -0.5)[0])
            a += c
        return z, torch.cat(o).reshape(x.shape[0], -1) @ self.w_out.t()

    def read(self, i):
        j = torch.arange(self.kept[i])
        slots = self.pages[i].cpu().long()[j // self.page] * self.page + j % self.page
        k, ka, v, va = self.at.esb.esb_kv4_unpack(self.b.cache, self.page, self.b.kv_heads, self.b.d, slots.cuda())
        return [(q.double() * a.double().repeat_interleave(32, 2)).cpu() for q, a in ((k, ka), (v, va))]


def near(y, want):
    assert float((y.cpu().double() - want).norm()) <= 0.10 * float(want.norm())


@pytest.mark.parametrize("heads,kv,d,dtype,norms", [(4, 2, 64, torch.bfloat16, True), (6, 1, 32, torch.float16, False),
                                                    (2, 2, 128, torch.bfloat16, True)])
def test_prompt_then_steps(at, heads, kv, d, dtype, norms):
    log("attention block heads=%d|%d d=%d" % (heads, kv, d))
    m = Model(at, heads, kv, d, dtype, norms)
    counts = [50, 1, 77]
    x, r, slots, pos, starts, lengths = m.batch(counts, 1)
    y, z = m.b.prompt(x.cuda(), r.cuda(), slots, pos, starts)
    assert y.dtype == z.dtype == dtype and y.shape == z.shape == x.shape
    rz, want = m.expected(x, r, pos, counts, False)
    decoder_ref.check_float(z, rz, 2.0 ** -24)
    near(y, want)
    # the prompt's keys in the cache are those of the block, within 4 bits (15 % as for weights) and its input's rounding
    k = m.read(2)[0]
    n = decoder_ref.rmsnorm(x, m.norm_weight, m.b.eps, r)[1]
    eps = 0.0 if not norms else at.D_EPS
    exact, _ = ref.turn((n @ m.w_qkv.t()).reshape(x.shape[0], -1, d)[:, heads:-kv], m.norms[1], eps, m.tab, pos.cpu(), False)
    assert float((k - exact[51:]).norm()) <= 0.18 * float(exact[51:].norm())
    for counts, seed in (([1, 1, 1], 2), ([1, 1, 1], 3), ([3, 0, 2], 4)):
        x, r, slots, pos, starts, lengths = m.batch(counts, seed)
        one = counts == [1, 1, 1]
        y, z = m.b.step(x.cuda(), r.cuda(), slots, pos, m.pages, lengths, None if one else starts)
        near(y, m.expected(x, r, pos, counts, True)[1])


def test_graph_of_steps(at):
    """A captured step, replayed for the tokens that follow: its inputs are copied into place."""
    a, b = (Model(at, 4, 2, 64, torch.bfloat16, True) for _ in range(2))
    for m in (a, b):
        x, r, slots, pos, starts, _ = m.batch([40, 9, 25], 1)
        m.b.prompt(x.cuda(), r.cuda(), slots, pos, starts)
    steps = [a.batch([1, 1, 1], s) for s in range(5, 10)]
    want = [a.b.step(x.cuda(), r.cuda(), slots, pos, a.pages, n) for x, r, slots, pos, _, n in steps]
    fixed = [t.cuda() for t in steps[0][:4]] + [steps[0][5].clone()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z = b.b.step(*fixed[:4], b.pages, fixed[4])
    for s, (wy, wz) in zip(steps, want):
        for to, t in zip(fixed, s[:4] + s[5:]):
            to.copy_(t)
        graph.replay()
        assert torch.equal(y, wy) and torch.equal(z, wz)
        torch.cuda.synchronize()
    assert torch.equal(a.b.cache, b.b.cache)


def test_refusals(at):
    w = at.synthetic(64, 2, 1, 32)
    table = ref.table(8, 32).cuda()
    for bad in (dict(w_qkv=w[0][:-1]), dict(w_out=w[1][:, 1:]), dict(q_norm=table[0]), dict(page=24)):
        with pytest.raises(ValueError):
            at.CachedAttention(**{**dict(w_qkv=w[0], w_out=w[1], heads=2, kv_heads=1, table=table, pages=2, page=16), **bad})


@pytest.mark.parametrize("heads,kv,d,dtype,norms", [(4, 2, 64, torch.bfloat16, True), (6, 1, 32, torch.float16, False)])
def test_prompts_and_steps_keep_the_same(at, heads, kv, d, dtype, norms):
    """The same tokens leave the same codes in the cache, as a prompt or as steps of many tokens."""
    a, b = (Model(at, heads, kv, d, dtype, norms) for _ in range(2))
    x, r, slots, pos, starts, lengths = a.batch([40, 9, 25], 1)
    a.b.prompt(x.cuda(), r.cuda(), slots, pos, starts)
    b.b.step(x.cuda(), r.cuda(), slots, pos, b.pages, lengths, starts)
    assert torch.equal(a.b.cache, b.b.cache)


def test_no_tokens(at):
    """A batch without tokens gives as many."""
    m = Model(at, 4, 2, 64, torch.bfloat16, True)
    x, r, slots, pos, starts, lengths = m.batch([0, 0, 0], 1)
    for out in (m.b.prompt(x.cuda(), r.cuda(), slots, pos, starts), m.b.step(x.cuda(), r.cuda(), slots, pos, m.pages, lengths, starts)):
        assert [tuple(t.shape) for t in out] == [tuple(x.shape)] * 2
