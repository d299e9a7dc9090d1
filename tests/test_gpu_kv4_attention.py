"""esb_kv4_attention against its definition in 64 bits on the cache's own values.

Tolerances: attention_ref.check, from the roundings that the operator makes: fp32 scores and sums,
p alpha in bf16 (2^-8) for bf16 outputs and in two bf16 (2^-17) for fp16, one rounding of the output.  With
more than 64 rows a sequence on average (queries x heads of a group) the probabilities are rounded to fp16
instead: 2^-11, and at least 2^-25."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
P_ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -16}


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


class Cache:
    """Sequences of random keys and values in shuffled pages; what no sequence owns holds NaN scales."""

    def __init__(self, esb, seed, lengths, heads, d, page, columns=None, spare=2, spread=0.3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-n // page) for n in lengths]
        total = sum(need) + spare
        self.esb, self.page, self.heads, self.d = esb, page, heads, d
        self.cache = torch.full((total, esb.esb_kv4_page_size(page, heads, d)), 0xFF, dtype=torch.uint8, device="cuda")
        order = torch.randperm(total, generator=g, device="cuda").int()
        self.columns = max(need + [1]) if columns is None else columns
        # entries behind a sequence's last key are nobody's page
        self.pages = torch.full((len(lengths), self.columns), 2 ** 30, dtype=torch.int32, device="cuda")
        at, slots = 0, []
        for i, n in enumerate(lengths):
            self.pages[i, :need[i]] = order[at:at + need[i]]
            j = torch.arange(n, device="cuda")
            slots.append(order[at:at + need[i]].long().repeat_interleave(page)[:n] * page + j % page)
            at += need[i]
        self.slots = slots
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        every = torch.cat(slots)
        n = every.numel()
        c = [torch.randint(0, 16, (n, heads, d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
        a = [(0.4 * torch.exp(spread * torch.randn(n, heads, d // 32, generator=g, device="cuda"))).to(torch.bfloat16)
             for _ in range(2)]
        esb.esb_kv4_pack(self.cache, page, c[0], a[0], c[1], a[1], every)

    def read(self, i):
        k, ka, v, va = self.esb.esb_kv4_unpack(self.cache, self.page, self.heads, self.d, self.slots[i])
        return [x.double() * a.double().repeat_interleave(32, 2) for x, a in ((k, ka), (v, va))]


def queries(seed, tokens, heads, d, dtype, size=0.6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(tokens, heads, d, generator=g, device="cuda")).to(dtype)


def verify(c, q, out, counts, scale=None, skip=()):
    at = 0
    many = -(-sum(counts) // len(counts)) * (q.shape[1] // c.heads) > 64
    for i, n in enumerate(counts):
        if i not in skip and n:
            k, v = c.read(i)
            m = k.shape[0]
            last = torch.arange(n) + m - n
            want = ref.attend(q[at:at + n], k, v, last, c.d ** -0.5 if scale is None else scale)
            p_round = 2.0 ** -11 if many else P_ROUND[q.dtype]
            ref.check(out[at:at + n], *want, keys=m, d=c.d, p_round=p_round, p_step=2.0 ** -25 if many else 0.0)
            for t in range(min(n, max(0, n - m))):
                assert not bool(out[at + t].any())
        at += n


LENGTHS = [1, 0, 16, 15, 17, 31, 33, 100, 128, 129, 300]


@pytest.mark.parametrize("kv,group", [(1, 1), (2, 3), (3, 4), (1, 16), (2, 17), (1, 40)])
@pytest.mark.parametrize("d,page", [(32, 16), (64, 16), (96, 32), (128, 64), (160, 16), (224, 128), (256, 16)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_one_token_each(esb, kv, group, d, page, t):
    log("kv4 decode kv=%d group=%d d=%d page=%d %s" % (kv, group, d, page, t))
    c = Cache(esb, d + group, LENGTHS, kv, d, page)
    q = queries(d, len(LENGTHS), kv * group, d, ref.TYPES[t])
    out = esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths)
    verify(c, q, out, [1] * len(LENGTHS))


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,page,length", [(2, 4, 128, 64, 9001), (1, 7, 64, 16, 20000), (1, 2, 256, 32, 3001),
                                                    (8, 1, 96, 128, 5000)])
def test_long_contexts(esb, t, kv, group, d, page, length):
    """Keys split over workgroups and joined; other sequences end in other parts."""
    lengths = [length, 1, 0, length // 3, 257, 128]
    log("kv4 long %s %d" % (t, length))
    c = Cache(esb, 3, lengths, kv, d, page)
    assert esb.esb_kv4_attention_workspace_size(6, kv * group, d, kv, 6, False, c.columns, page) > 0
    q = queries(4, 6, kv * group, d, ref.TYPES[t])
    out = esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths)
    verify(c, q, out, [1] * 6)
    # the same call gives the same bits, in its own workspace too
    need = esb.esb_kv4_attention_workspace_size(6, kv * group, d, kv, 6, False, c.columns, page)
    ws = torch.full((need + 100,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(out, esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths, workspace=ws))
    assert bool((ws[need:] == 0xFF).all())


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,page", [(1, 1, 64, 16), (2, 7, 64, 16), (2, 4, 128, 64), (1, 5, 96, 32), (1, 3, 256, 16)])
@pytest.mark.parametrize("counts,lengths", [([1, 5, 0, 3], [1, 5, 7, 700]), ([2, 64, 17], [40, 64, 1000]),
                                            ([200, 1, 0, 0, 33], [200, 2000, 0, 5, 34]), ([300, 129], [4000, 6001]),
                                            ([5, 9, 4], [3, 0, 4])])       # fewer keys than queries
def test_several_tokens(esb, t, kv, group, d, page, counts, lengths):
    log("kv4 tokens=%s lengths=%s kv=%d group=%d d=%d %s" % (counts, lengths, kv, group, d, t))
    c = Cache(esb, 5, lengths, kv, d, page)
    tokens = sum(counts)
    q = queries(6, tokens + 3, kv * group, d, ref.TYPES[t])
    starts = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.5)
    got = esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths, starts=starts, out=out)
    assert got is out
    verify(c, q, out, counts)
    assert bool((out[tokens:] == 7.5).all())          # rows behind the last sequence


def test_many_sequences(esb):
    """More sequences than a wave has lanes, most of them without a token now."""
    counts = [(3 * i) % 5 if i % 3 else 0 for i in range(150)]
    lengths = [c + (7 * i) % 90 for i, c in enumerate(counts)]
    c = Cache(esb, 8, lengths, 2, 64, 16)
    q = queries(9, sum(counts), 6, 64, torch.bfloat16)
    starts = torch.tensor([sum(counts[:i]) for i in range(151)], dtype=torch.int32, device="cuda")
    out = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths, starts=starts)
    verify(c, q, out, counts)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_sharp_and_growing_scores(esb, t):
    """Softmaxes of one key, and a maximum that moves by much many times."""
    lengths = [700, 700]
    c = Cache(esb, 10, lengths, 1, 128, 16, spread=1.5)
    q = queries(11, 2, 8, 128, ref.TYPES[t], size=8.0)
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, scale=0.5)
    verify(c, q, out, [1, 1], scale=0.5)
    # keys that grow: alpha doubles every 32 keys
    codes = torch.full((700, 1, 128), 0, dtype=torch.uint8, device="cuda")
    a = (2.0 ** (torch.arange(700, device="cuda") // 64)).to(torch.bfloat16)[:, None, None].expand(700, 1, 4).contiguous()
    va = torch.ones_like(a)
    vc = torch.randint(0, 16, (700, 1, 128), device="cuda", dtype=torch.uint8)
    esb.esb_kv4_pack(c.cache, 16, codes, a, vc, va, c.slots[0])
    q = queries(12, 2, 8, 128, ref.TYPES[t], size=0.05).abs()
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, scale=0.5)
    verify(c, q, out, [1, 1], scale=0.5)


def test_large_scales_in_fp16(esb):
    """Scales beyond fp16 in keys whose scores are small, values near its end."""
    c = Cache(esb, 13, [50], 1, 64, 16)
    k = torch.randint(0, 16, (50, 1, 64), device="cuda", dtype=torch.uint8)
    a = torch.full((50, 1, 2), 1e6, device="cuda").to(torch.bfloat16)
    va = torch.full((50, 1, 2), 9000.0, device="cuda").to(torch.bfloat16)
    esb.esb_kv4_pack(c.cache, 16, k, a, k, va, c.slots[0])
    q = (queries(14, 1, 2, 64, torch.float16) * 1e-5).to(torch.float16)
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths)
    verify(c, q, out, [1])
    # as a prompt, both types, queries far below and above 1
    for dtype, size in ((torch.float16, 1e-5), (torch.bfloat16, 1e-30), (torch.bfloat16, 1e5)):
        a = torch.full((50, 1, 2), 1e6 if size < 1 else 1e-4, device="cuda").to(torch.bfloat16)
        a[7] = a[7] * 64
        esb.esb_kv4_pack(c.cache, 16, k, a * (1e25 if size < 1e-20 else 1), k, va, c.slots[0])
        q = (queries(15, 50, 4, 64, torch.float32) * size).to(dtype)
        out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=torch.tensor([0, 50], dtype=torch.int32, device="cuda"))
        verify(c, q, out, [50])


def test_value_scales_that_grow(esb):
    """Value scales over many powers of two along the keys, as the prompt form brings them to one."""
    n = 500
    c = Cache(esb, 33, [n], 1, 128, 16)
    g = torch.Generator(device="cuda").manual_seed(34)
    codes = torch.randint(0, 16, (n, 1, 128), generator=g, device="cuda", dtype=torch.uint8)
    q = queries(35, n, 4, 128, torch.bfloat16)
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for shift in (torch.arange(n) // 20 - 12, 12 - torch.arange(n) // 20, torch.zeros(n)):
        a = (0.4 * 2.0 ** shift.cuda().double())[:, None, None].expand(n, 1, 4).to(torch.bfloat16).contiguous()
        esb.esb_kv4_pack(c.cache, 16, codes, torch.full_like(a, 0.3), codes, a, c.slots[0])
        out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts)
        verify(c, q, out, [n])


@pytest.mark.parametrize("group", [1, 2, 16])      # by how many rows share keys: each kernel
@pytest.mark.parametrize("d", [64, 96, 256])
def test_not_finite(esb, group, d):
    """NaN scales reach the queries that see them, and no others; NaN queries themselves only."""
    counts, lengths = [40, 1], [60, 30]
    c = Cache(esb, 15, lengths, 1, d, 16)
    q = queries(16, 41, group, d, torch.bfloat16)
    starts = torch.tensor([0, 40, 41], dtype=torch.int32, device="cuda")
    clean = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts)
    for which in (0, 1):
        codes = torch.zeros(1, 1, d, dtype=torch.uint8, device="cuda")
        nan = torch.full((1, 1, d // 32), float("nan"), dtype=torch.bfloat16, device="cuda")
        one = torch.ones_like(nan)
        c = Cache(esb, 15, lengths, 1, d, 16)
        # key 45 of sequence 0 is seen by its queries 25 ..
        esb.esb_kv4_pack(c.cache, 16, codes, nan if which == 0 else one, codes, nan if which else one, c.slots[0][45:46])
        out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts)
        assert torch.equal(out[:25], clean[:25]) and torch.equal(out[40:], clean[40:])
        assert bool(torch.isnan(out[25:40]).all())
    q[3, group - 1, 5] = float("nan")
    q[40, 0, 0] = float("inf")
    c = Cache(esb, 15, lengths, 1, d, 16)
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts)
    assert bool(torch.isnan(out[3, group - 1]).all()) and bool(torch.isnan(out[40, 0]).all())
    keep = torch.ones(41, group, dtype=torch.bool)
    keep[3, group - 1] = keep[40, 0] = False
    assert torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("columns", [None, 700])
def test_bad_lengths_and_pages(esb, columns):
    """Lengths beyond the page table and pages that are not the cache's give NaN, and read nothing.  With many
    columns the keys are split over workgroups."""
    lengths = [100, 90, 80, 70]
    c = Cache(esb, 17, lengths, 2, 64, 16, columns=columns)
    q = queries(18, 4, 4, 64, torch.bfloat16)
    clean = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths)
    c.lengths[0] = c.columns * 16 + 1
    c.lengths[3] = -5
    for page in (-1, c.cache.shape[0], 2 ** 31 - 1):
        c.pages[2, 3] = page
        out = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths)
        assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[2]).all())
        assert not bool(out[3].any()) and torch.equal(out[1], clean[1])


def test_starts_of_anything(esb):
    """Starts that do not ascend or leave the tokens read and write nothing outside."""
    lengths = [100, 90, 80]
    c = Cache(esb, 19, lengths, 2, 64, 16)
    q = queries(20, 30, 4, 64, torch.bfloat16)
    buf = torch.full((50, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    for s in ([0, -5, 40, 7], [10, 5, 2, 0], [2 ** 31 - 1, 0, 9, 2 ** 31 - 1], [-2 ** 31, 20, 10, 30]):
        starts = torch.tensor(s, dtype=torch.int32, device="cuda")
        esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths, starts=starts, out=buf[10:40])
        assert bool((buf[:10] == 3.0).all()) and bool((buf[40:] == 3.0).all())


@pytest.mark.parametrize("shift", [0, 1])
def test_pitches(esb, shift):
    c = Cache(esb, 21, [77, 200], 2, 96, 16)
    q = queries(22, 2, 6, 96, torch.float16)
    want = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths)
    buf = torch.full((2 * 900 + 9,), 5.0, dtype=torch.float16, device="cuda")
    v = buf.as_strided((2, 6, 96), (900, 100, 1), shift)
    v.copy_(q)
    ob = torch.full((6 * 300 + 9,), 5.0, dtype=torch.float16, device="cuda")
    o = ob.as_strided((2, 6, 96), (97, 300, 1), shift)      # heads before tokens
    pages = torch.full((2, c.columns + 3), -7, dtype=torch.int32, device="cuda")
    pages[:, :c.columns] = c.pages
    esb.esb_kv4_attention(v, c.cache, 16, 2, pages[:, :c.columns], c.lengths, out=o)
    assert torch.equal(o, want)
    o.fill_(5.0)
    assert bool((ob == 5.0).all())


def test_far_pages(esb):
    """Offsets beyond 2^32 bytes in the cache."""
    heads, d, page = 8, 128, 4096
    size = esb.esb_kv4_page_size(page, heads, d)
    pages = 2 ** 32 // size + 3
    small = Cache(esb, 23, [page + 50], heads, d, page, spare=0)
    cache = torch.empty(pages, size, dtype=torch.uint8, device="cuda")
    far = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    cache[far[0].long()] = small.cache[small.pages[0].long()]
    q = queries(24, 1, 16, d, torch.bfloat16)
    want = esb.esb_kv4_attention(q, small.cache, page, heads, small.pages, small.lengths)
    assert torch.equal(esb.esb_kv4_attention(q, cache, page, heads, far, small.lengths), want)


def test_graphs_share_a_workspace(esb):
    """Two captured calls over one workspace, replayed in turn with eager calls between."""
    lengths = [3000, 1700, 5]
    c = Cache(esb, 25, lengths, 2, 128, 64)
    qs = [queries(s, 3, 8, 128, torch.bfloat16) for s in (26, 27, 28)]
    want = [esb.esb_kv4_attention(q, c.cache, 64, 2, c.pages, c.lengths) for q in qs]
    need = esb.esb_kv4_attention_workspace_size(3, 8, 128, 2, 3, False, c.columns, 64)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs, ins, outs = [], [qs[0].clone(), qs[1].clone()], []
    torch.cuda.synchronize()
    for x in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(esb.esb_kv4_attention(x, c.cache, 64, 2, c.pages, c.lengths, workspace=ws))
        graphs.append(g)
    for turn in range(4):
        a, b = turn % 3, (turn + 1) % 3
        ins[0].copy_(qs[a]), ins[1].copy_(qs[b])
        graphs[0].replay()
        graphs[1].replay()
        eager = esb.esb_kv4_attention(qs[2], c.cache, 64, 2, c.pages, c.lengths, workspace=ws)
        assert torch.equal(outs[0], want[a]) and torch.equal(outs[1], want[b]) and torch.equal(eager, want[2])
        torch.cuda.synchronize()


def test_binding_refusals(esb):
    c = Cache(esb, 29, [40, 9], 2, 64, 16)
    q = queries(30, 2, 4, 64, torch.bfloat16)
    call = dict(q=q, cache=c.cache, page=16, kv_heads=2, pages=c.pages, lengths=c.lengths)
    for bad in (dict(q=q[:, :, :32]), dict(cache=c.cache[:, 1:]), dict(pages=c.pages[:1]), dict(pages=c.pages.long()),
                dict(out=q[:, :2]), dict(out=q.half()), dict(workspace=torch.zeros(2, 8, device="cuda")[:, 1:]),
                dict(starts=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            esb.esb_kv4_attention(**{**call, **bad})
    for bad in (dict(lengths=c.lengths.long()), dict(lengths=c.lengths.cpu()), dict(q=q.double())):
        with pytest.raises(TypeError):
            esb.esb_kv4_attention(**{**call, **bad})
    for bad in (dict(q=q[:, :3]), dict(q=q.float()), dict(out=q), dict(scale=0.0), dict(kv_heads=0)):
        with pytest.raises((esb.EsbError, ValueError)):
            esb.esb_kv4_attention(**{**call, **bad})


def test_streams(esb):
    c = Cache(esb, 31, [5000, 40], 2, 128, 64)
    q = queries(32, 2, 8, 128, torch.bfloat16)
    want = esb.esb_kv4_attention(q, c.cache, 64, 2, c.pages, c.lengths)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for given in (s, s.cuda_stream):
        with torch.cuda.stream(s):
            y = q.float().to(torch.bfloat16)
        out = esb.esb_kv4_attention(y, c.cache, 64, 2, c.pages, c.lengths, stream=given)
        s.synchronize()
        assert torch.equal(out, want)


def wide(seqs, heads, counts, group, d, page):
    """Columns of a page table over which a call's work is shared evenly, whatever tile it takes: at least 20480
    steps of 128 keys where each sequence has one tile of rows."""
    return 128 // page * (-(-20480 // (seqs * heads)) + 32) if page <= 128 else 20480 // (seqs * heads) + 32


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,page", [(1, 1, 32, 16), (2, 4, 128, 64), (1, 7, 64, 16), (3, 12, 64, 32),
                                             (1, 40, 128, 64), (2, 3, 96, 128), (1, 20, 96, 16), (2, 2, 256, 16),
                                             (1, 4, 160, 64), (1, 30, 64, 64)])
@pytest.mark.parametrize("many", [False, True])
def test_even_shares(esb, t, kv, group, d, page, many):
    """Work that workgroups share evenly: sequences that end inside a share, take several, have no token or no key;
    fewer and more sequences than a wave has lanes, one of them longer than all others."""
    seqs = 150 if many else 13
    lengths = [(53 * i) % 400 if i % 5 else (i // 5) % 3 for i in range(seqs)]
    lengths[seqs // 2], lengths[-1] = 2600, 129
    c = Cache(esb, 70, lengths, kv, d, page, columns=wide(seqs, kv, 1, group, d, page))
    q = queries(71, seqs, kv * group, d, ref.TYPES[t])
    verify(c, q, esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths), [1] * seqs)
    counts = [(7 * i) % 4 for i in range(seqs)]
    q = queries(72, sum(counts) + 3, kv * group, d, ref.TYPES[t])
    starts = torch.tensor([sum(counts[:i]) for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths, starts=starts, out=out)
    verify(c, q, out, counts)
    assert bool((out[sum(counts):] == 3.0).all())


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,page", [(2, 4, 128, 64), (1, 7, 64, 16), (1, 1, 32, 16), (2, 3, 96, 32)])
@pytest.mark.parametrize("size", [40, 130])
def test_even_shares_of_many_rows(esb, t, kv, group, d, page, size):
    """Parts of prompts, some empty, some without keys before them, over a table of many columns."""
    counts = [size, 0, 3 * size, 1, 2 * size + 7, size // 2]
    counts = [n * 4 // group if n > 1 else n for n in counts]
    lengths = [n + k for n, k in zip(counts, [700, 5, 0, 300, 1100, 64])]
    lengths[5] = max(counts[5] - 9, 0)      # the first tokens see nothing
    c = Cache(esb, 79, lengths, kv, d, page, columns=400000 // page)
    q = queries(80, sum(counts) + 3, kv * group, d, ref.TYPES[t])
    starts = torch.tensor([sum(counts[:i]) for i in range(7)], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths, starts=starts, out=out)
    verify(c, q, out, counts)
    assert bool((out[sum(counts):] == 3.0).all())


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,page", [(1, 96, 64, 16), (2, 65, 128, 64), (1, 200, 96, 32), (1, 300, 256, 64)])
@pytest.mark.parametrize("columns", [None, 4096])
def test_large_groups(esb, t, kv, group, d, page, columns):
    """One query a sequence, whose heads alone are many rows."""
    lengths = [1, 0, 65, 700, 64, 2000, 129]
    c = Cache(esb, 81, lengths, kv, d, page, columns=columns)
    q = queries(82, len(lengths), kv * group, d, ref.TYPES[t])
    verify(c, q, esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths), [1] * len(lengths))


def test_even_shares_of_anything(esb):
    """The same over bad lengths and pages, and starts that do not ascend or leave the tokens."""
    lengths = [100, 90, 700, 70]
    c = Cache(esb, 73, lengths, 2, 128, 16, columns=wide(4, 2, 1, 8, 128, 16))
    q = queries(74, 4, 16, 128, torch.bfloat16)
    clean = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths)
    c.lengths[0] = c.columns * 16 + 1
    c.lengths[3] = -5
    for page in (-1, c.cache.shape[0], 2 ** 31 - 1):
        c.pages[2, 30] = page
        out = esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths)
        assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[2]).all())
        assert not bool(out[3].any())
        # cut elsewhere: probabilities rounded under another maximum (twice 2^-9 of a mean of |v|, which is below
        # 2: codes of 1.9 on average, scales about 0.4), and a bf16 step of the output
        torch.testing.assert_close(out[1], clean[1], rtol=2.0 ** -7, atol=2.0 ** -7)
    q = queries(75, 30, 16, 128, torch.bfloat16)
    buf = torch.full((50, 16, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    for s in ([0, -5, 40, 7, 30], [10, 5, 2, 0, 0], [2 ** 31 - 1, 0, 9, 2 ** 31 - 1, 5], [-2 ** 31, 20, 10, 30, 30],
              [0, 30, 0, 30, 0], [-9, -7, -2, 5, 2 ** 31 - 1]):
        starts = torch.tensor(s, dtype=torch.int32, device="cuda")
        esb.esb_kv4_attention(q, c.cache, 16, 2, c.pages, c.lengths, starts=starts, out=buf[10:40])
        assert bool((buf[:10] == 3.0).all()) and bool((buf[40:] == 3.0).all())


def test_even_shares_in_graphs(esb):
    """Two captured calls that share work evenly over one workspace; the lengths change between replays."""
    seqs = 9
    lengths = [300 * i + 40 for i in range(seqs)]
    c = Cache(esb, 76, lengths, 2, 128, 64, columns=wide(seqs, 2, 1, 8, 128, 64))
    qs = [queries(s, seqs, 16, 128, torch.bfloat16) for s in (77, 78)]
    need = esb.esb_kv4_attention_workspace_size(seqs, 16, 128, 2, seqs, False, c.columns, 64)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    now = c.lengths.clone()
    graphs, outs = [], []
    esb.esb_kv4_attention(qs[0], c.cache, 64, 2, c.pages, now, workspace=ws)
    torch.cuda.synchronize()
    for x in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(esb.esb_kv4_attention(x, c.cache, 64, 2, c.pages, now, workspace=ws))
        graphs.append(g)
    for turn in range(4):
        now.copy_((c.lengths - 13 * turn * torch.arange(seqs, device="cuda")).int())
        graphs[0].replay()
        graphs[1].replay()
        for x, out in zip(qs, outs):
            assert torch.equal(out, esb.esb_kv4_attention(x, c.cache, 64, 2, c.pages, now))
        torch.cuda.synchronize()
