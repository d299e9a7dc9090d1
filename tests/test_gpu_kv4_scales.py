"""esb_kv4_attention where queries, keys and values lie far apart: zeros, the least scales, and scales of
one key, value or group far above another's, seen or not.

Tolerances: those of test_gpu_kv4_attention, which say nothing of a range; what lies behind a query's last
key enters none of them."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log
from test_gpu_kv4_attention import Cache, esb, queries, verify, wide  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def starts(counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


# query heads of a key head, by how many rows 40 queries make, or one: each kernel
FEW, SOME, MANY = (1, None), (1, 40), (8, 40)


@pytest.mark.parametrize("group,n", [(4, None), SOME, MANY, (32, 40)])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (160, 16), (256, 16)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("columns", [None, 4096])
def test_zeros(esb, group, n, d, page, t, columns):  # noqa: F811
    """Zero and tiny queries over keys of zeros, in a cache of zeros and appended: the mean of what is seen."""
    counts, lengths = [n or 1, 1], [77, 40]
    for appended in (False, True):
        for size in (0.0, 1e-30 if t == "bf16" else 1e-7, 0.6):
            log("kv4 zeros group=%d n=%s d=%d %s appended=%d size=%g" % (group, n, d, t, appended, size))
            c = Cache(esb, 1, lengths, 2, d, page, columns=columns)
            every = torch.cat(c.slots)
            v = queries(2, every.numel(), 2, d, BF16)
            if appended:
                esb.esb_kv4_append(c.cache, page, torch.zeros_like(v), v, every)
            else:
                _, _, codes, alpha = esb.esb_kv4_unpack(c.cache, page, 2, d, every)
                zero = torch.zeros(every.numel(), 2, d, dtype=torch.uint8, device="cuda")
                esb.esb_kv4_pack(c.cache, page, zero, torch.zeros_like(alpha), zero + 3, alpha, every)
            q = queries(3, sum(counts), 2 * group, d, ref.TYPES[t], size=size)
            out = esb.esb_kv4_attention(q, c.cache, page, 2, c.pages, c.lengths, starts=starts(counts))
            verify(c, q, out, counts)


def test_tiny_products(esb):  # noqa: F811
    """Queries, keys and a scale whose products all but vanish."""
    c = Cache(esb, 4, [90], 1, 128, 16)
    every = c.slots[0]
    k, v = queries(5, 90, 1, 128, BF16, size=1e-15), queries(6, 90, 1, 128, BF16)
    esb.esb_kv4_append(c.cache, 16, k, v, every)
    for size, scale in ((1e-15, None), (1e-30, None), (1.0, 1e-30), (1e-30, 1e-38)):
        q = queries(7, 40, 4, 128, BF16, size=size)
        out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([40]), scale=scale)
        verify(c, q, out, [40], scale=scale)


LEAST = 2.0 ** -126


def verify_rows(c, q, out, rows, scale=None, at=0, many=None):
    """Those rows of sequence `at`, whose queries q are, by what they see.  A weight below fp32's smallest normal
    number, beside a largest one of at least 1, may count as zero: that is LEAST of the sum of |v|."""
    k, v = c.read(at)
    n = q.shape[0]
    last = torch.arange(n) + k.shape[0] - n
    rows = torch.as_tensor(rows)
    m = int(last[rows].max()) + 1
    many = n * (q.shape[1] // c.heads) > 64 if many is None else many
    want = ref.attend(q[rows], k[:m], v[:m], last[rows], c.d ** -0.5 if scale is None else scale)
    p_round = 2.0 ** -11 if many else 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -16
    ref.check(out[rows], *want, keys=m, d=c.d, p_round=p_round, p_step=2.0 ** -25 if many else LEAST)


@pytest.mark.parametrize("power", [10, 18, 24, 32, 60])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 16)])
@pytest.mark.parametrize("group,n", [FEW, SOME, MANY, (16, None)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("columns", [None, 8192])
def test_large_scores(esb, power, d, page, group, n, t, columns):  # noqa: F811
    """Scores of about 2^power, finite: the largest takes all, and nothing is NaN.  The queries before a row of such
    scores, and heads beside it, are as they were."""
    c = Cache(esb, 80, [300], 1, d, page, columns=columns)
    g = torch.Generator(device="cuda").manual_seed(81)
    codes = [torch.randint(0, 16, (300, 1, d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    a = (0.4 * torch.exp(0.3 * torch.randn(300, 1, d // 32, generator=g, device="cuda"))).to(BF16)
    esb.esb_kv4_pack(c.cache, page, codes[0], (a.double() * 2.0 ** power).to(BF16), codes[1], a, c.slots[0])
    q = queries(82, n or 1, group, d, ref.TYPES[t])
    call = lambda q: esb.esb_kv4_attention(q, c.cache, page, 1, c.pages, c.lengths, starts=starts([n or 1]))  # noqa: E731
    verify_rows(c, q, call(q), range(n or 1))
    q[:, :, :] = (q.double() * 2.0 ** -min(power, 12)).to(q.dtype)
    want = call(q)
    far = q.clone()
    far[-1, -1] = 30000.0
    out = call(far)
    assert bool(torch.isfinite(out).all())
    assert torch.equal(out.flatten(0, 1)[:-1], want.flatten(0, 1)[:-1])


def spread(esb, c, seed, alpha_k, alpha_v):  # noqa: F811
    """Keys and values of sequence 0 with the given scales (tokens x heads x groups)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = c.slots[0].numel()
    k, v = (torch.randint(0, 16, (n, c.heads, c.d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    esb.esb_kv4_pack(c.cache, c.page, k, alpha_k.to(BF16), v, alpha_v.to(BF16), c.slots[0])


@pytest.mark.parametrize("power", [13, 20, 24, 30, 40, 100])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("group,n", [SOME, MANY])
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("columns", [None, 8192])
def test_large_scales_out_of_sight(esb, power, what, d, page, group, n, t, columns):  # noqa: F811
    """A later key or value that is 2^power times the others does not reach the queries before it."""
    log("kv4 out of sight 2^%d %s d=%d group=%d %s columns=%s" % (power, what, d, group, t, columns))
    for before in (30, 333):                # a first tile of keys, and after several
        c = Cache(esb, 40, [before + n], 1, d, page, columns=columns)
        g = torch.Generator(device="cuda").manual_seed(41)
        a = [0.4 * torch.exp(0.3 * torch.randn(before + n, 1, d // 32, generator=g, device="cuda")) for _ in range(2)]
        at = before + n - 9                 # the last nine queries see it
        a[what == "v"][at] *= 2.0 ** power
        spread(esb, c, 42, *a)
        q = queries(43, n, group, d, ref.TYPES[t])
        out = esb.esb_kv4_attention(q, c.cache, page, 1, c.pages, c.lengths, starts=starts([n]))
        verify_rows(c, q, out, range(n - 9))
        if t == "bf16":
            verify_rows(c, q, out, range(n))


@pytest.mark.parametrize("power", [16, 24, 40, 100, -24, -60])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (224, 16)])
@pytest.mark.parametrize("group,n", [FEW, SOME, MANY])
def test_groups_far_apart(esb, power, what, d, page, group, n):  # noqa: F811
    """One scale group of a head 2^power times the others: each keeps its bits."""
    log("kv4 groups 2^%d %s d=%d group=%d n=%s" % (power, what, d, group, n))
    c = Cache(esb, 50, [200], 1, d, page)
    g = torch.Generator(device="cuda").manual_seed(51)
    a = [0.4 * torch.exp(0.3 * torch.randn(200, 1, d // 32, generator=g, device="cuda")) for _ in range(2)]
    a[what == "v"][:, :, 1] *= 2.0 ** power
    spread(esb, c, 52, *a)
    q = queries(53, n or 1, group, d, BF16)
    if what == "k":
        q[:, :, 32:64] *= 2.0 ** -min(abs(power), 60) if power > 0 else 1      # scores that the other groups decide
    out = esb.esb_kv4_attention(q, c.cache, page, 1, c.pages, c.lengths, starts=starts([n or 1]))
    verify_rows(c, q, out, range(n or 1))


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 16)])
@pytest.mark.parametrize("columns", [None, 8192])
def test_keys_far_apart(esb, d, page, columns):  # noqa: F811
    """Scales of keys and values anywhere over 2^80, seen by all; queries whose elements are as far apart."""
    c = Cache(esb, 60, [300], 1, d, page, columns=columns)
    g = torch.Generator(device="cuda").manual_seed(61)
    for wide_q in (False, True):
        a = [2.0 ** torch.randint(-60, 20, (300, 1, d // 32), generator=g, device="cuda").double() for _ in range(2)]
        spread(esb, c, 62, *a)
        q = queries(63, 40, 8, d, torch.float32)
        if wide_q:
            q = q * 2.0 ** torch.randint(-60, 1, q.shape, generator=g, device="cuda").float()
        out = esb.esb_kv4_attention(q.to(BF16), c.cache, page, 1, c.pages, c.lengths, starts=starts([40]))
        verify_rows(c, q.to(BF16), out, range(40))


def test_zero_tokens_among_others(esb):  # noqa: F811
    """Appended zeros have the least scale of all, beside ordinary keys and values."""
    n, d = 200, 128
    c = Cache(esb, 64, [n], 1, d, 16)
    k, v = queries(65, n, 1, d, BF16), queries(66, n, 1, d, BF16)
    k[50:90], v[70:120] = 0, 0
    k[130, :, 32:64], v[131, :, 64:] = 0, 0
    esb.esb_kv4_append(c.cache, 16, k, v, c.slots[0])
    q = queries(67, 60, 4, d, BF16)
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([60]))
    verify(c, q, out, [60])


def test_far_apart_in_graphs(esb):  # noqa: F811
    """A captured call whose cache takes the usual way in one replay and the other in the next."""
    c = Cache(esb, 90, [400], 1, 128, 16, columns=8192)
    g = torch.Generator(device="cuda").manual_seed(91)
    a = 0.4 * torch.exp(0.3 * torch.randn(400, 1, 4, generator=g, device="cuda"))
    spread(esb, c, 92, a, a)
    near = c.cache.clone()
    a[380, 0, 2] *= 2.0 ** 40
    a[3, 0, 1] *= 2.0 ** -50
    spread(esb, c, 92, a, a)
    caches = [near, c.cache.clone()]
    q = queries(93, 40, 8, 128, BF16)
    st = starts([40])
    want = [esb.esb_kv4_attention(q, x, 16, 1, c.pages, c.lengths, starts=st) for x in caches]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=st)
    for turn in range(5):
        c.cache.copy_(caches[turn % 2])
        graph.replay()
        assert torch.equal(out, want[turn % 2])
        torch.cuda.synchronize()
        verify_rows(c, q, out, range(40))


@pytest.mark.parametrize("power", [100, 118, 121, 124])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 16)])
@pytest.mark.parametrize("group,n", [FEW, SOME, MANY, (16, None), (32, None)])
@pytest.mark.parametrize("columns", [None, 8192])
def test_largest_values(esb, power, d, page, group, n, columns):  # noqa: F811
    """Values near the end of bf16 under weights that grow by less than 2^8: outputs are finite, and so are the sums."""
    log("kv4 largest values 2^%d d=%d group=%d n=%s columns=%s" % (power, d, group, n, columns))
    m = 700 if columns else 150
    c = Cache(esb, 70, [m], 1, d, page, columns=columns)
    codes = torch.full((m, 1, d), 0, dtype=torch.uint8, device="cuda")      # ones
    up = torch.arange(m, device="cuda").float() / m
    a = up[:, None, None].expand(m, 1, d // 32).to(BF16).contiguous()
    # one value in 60 is large, or sums of 700 would leave fp32 themselves
    va = torch.where(torch.arange(m, device="cuda") % 60 == 7, 2.0 ** power, 2.0 ** (power - 9))
    va = va[:, None, None].expand(m, 1, d // 32).to(BF16).contiguous()
    esb.esb_kv4_pack(c.cache, page, codes, a, codes, va, c.slots[0])
    # scores from 0 to 5.4 (log2: 7.8)
    q = torch.full((n or 1, group, d), 5.4 / d, dtype=BF16, device="cuda")
    out = esb.esb_kv4_attention(q, c.cache, page, 1, c.pages, c.lengths, starts=starts([n or 1]), scale=1.0)
    verify_rows(c, q, out, range(n or 1), scale=1.0)


@pytest.mark.parametrize("group,n", [FEW, SOME, MANY])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 96])
def test_infinite_scales(esb, group, n, what, value, d):  # noqa: F811
    """Packed infinities are kept as NaN: whoever sees one gets NaN, from every kernel alike."""
    c = Cache(esb, 94, [100], 1, d, 16)
    q = queries(95, n or 1, group, d, BF16)
    clean = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([n or 1]))
    codes = torch.randint(0, 16, (1, 1, d), device="cuda", dtype=torch.uint8)
    a = torch.full((1, 1, d // 32), value, dtype=BF16, device="cuda")
    at = 99 if n is None else 80            # seen by the only query, or by those from 20 on
    esb.esb_kv4_pack(c.cache, 16, codes, a if what == "k" else torch.ones_like(a), codes, a if what == "v" else torch.ones_like(a),
                     c.slots[0][at:at + 1])
    _, ka, _, va = esb.esb_kv4_unpack(c.cache, 16, 1, d, c.slots[0][at:at + 1])
    assert bool(torch.isnan(ka if what == "k" else va).all())
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([n or 1]))
    first = 0 if n is None else 20
    assert torch.equal(out[:first], clean[:first]) and bool(torch.isnan(out[first:]).all())


@pytest.mark.parametrize("kv,group,d,page", [(1, 1, 32, 16), (2, 4, 128, 64), (1, 7, 64, 16), (3, 12, 64, 32), (1, 40, 128, 64),
                                             (2, 2, 256, 16), (1, 30, 96, 64), (1, 90, 128, 64), (1, 70, 64, 16)])
@pytest.mark.parametrize("several", [False, True])
def test_far_apart_in_even_shares(esb, kv, group, d, page, several):  # noqa: F811
    """The same in work that workgroups share evenly: beside ordinary sequences some whose values are near the end
    of bf16, some whose scales are far apart, some of zeros; items that begin and end in any share."""
    seqs = 13
    lengths = [(53 * i) % 400 + 5 for i in range(seqs)]
    lengths[6] = 2600
    counts = [1 + (7 * i) % 4 if several else 1 for i in range(seqs)]
    c = Cache(esb, 96, lengths, kv, d, page, columns=wide(seqs, kv, 1, group, d, page))
    g = torch.Generator(device="cuda").manual_seed(97)
    for i in range(seqs):
        if i % 4 == 3:
            continue
        n, ones = lengths[i], torch.ones(lengths[i], kv, d // 32, device="cuda")
        codes = [torch.randint(0, 16, (n, kv, d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
        a, va = 0.3 * ones, 0.4 * ones
        if i % 4 == 0:          # weights that grow by less than 2^8
            codes = [torch.zeros_like(x) for x in codes]
            a = ones * (torch.arange(n, device="cuda") / n)[:, None, None]
            va = ones * torch.where(torch.arange(n, device="cuda") % 90 == 7, 2.0 ** 122, 2.0 ** 110)[:, None, None]
        elif i % 4 == 1:
            a, va = (x * 2.0 ** torch.randint(-40, 1, x.shape, generator=g, device="cuda") for x in (a, va))
        else:
            codes, a, va = [torch.full_like(x, 6) for x in codes], 2.0 ** -126 * ones, 2.0 ** -126 * ones
        esb.esb_kv4_pack(c.cache, page, codes[0], a.to(BF16), codes[1], va.to(BF16), c.slots[i])
    q = queries(98, sum(counts), kv * group, d, BF16)
    at = [sum(counts[:i]) for i in range(seqs)]
    for i in range(0, seqs, 4):
        q[at[i]:at[i] + counts[i]] = 5.4 / d
    st = starts(counts) if several else None
    out = esb.esb_kv4_attention(q, c.cache, page, kv, c.pages, c.lengths, starts=st, scale=1.0)
    many = -(-sum(counts) // seqs) * group > 64
    for i in range(seqs):
        verify_rows(c, q[at[i]:at[i] + counts[i]], out[at[i]:at[i] + counts[i]], range(counts[i]), scale=1.0, at=i, many=many)
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("group,n", [FEW, SOME, MANY])
@pytest.mark.parametrize("power", [10, 40])
def test_large_negative_scores(esb, group, n, power):  # noqa: F811
    c = Cache(esb, 99, [200], 1, 64, 16)
    codes = torch.randint(0, 6, (200, 1, 64), device="cuda", dtype=torch.uint8, generator=torch.Generator(device="cuda").manual_seed(1))
    a = torch.full((200, 1, 2), 2.0 ** power, device="cuda").to(BF16)
    esb.esb_kv4_pack(c.cache, 16, codes, a, codes, torch.ones_like(a), c.slots[0])
    q = -queries(100, n or 1, group, 64, BF16).abs()
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([n or 1]))
    verify_rows(c, q, out, range(n or 1))


@pytest.mark.parametrize("group,n", [FEW, SOME, MANY, (16, None)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("columns", [None, 8192])
@pytest.mark.parametrize("at", [0, 96, 200, 640])
def test_large_negative_scores_beside_others(esb, group, n, d, columns, at):  # noqa: F811
    """Runs of keys whose scores are about -2^40 have no weight beside ordinary ones."""
    c = Cache(esb, 101, [700], 1, d, 16, columns=columns)
    g = torch.Generator(device="cuda").manual_seed(102)
    codes = torch.randint(0, 6, (700, 1, d), device="cuda", dtype=torch.uint8, generator=g)
    v = torch.randint(0, 16, (700, 1, d), device="cuda", dtype=torch.uint8, generator=g)
    a = 0.1 * torch.exp(0.3 * torch.randn(700, 1, d // 32, device="cuda", generator=g))
    a[at:at + 150] *= 2.0 ** 40
    esb.esb_kv4_pack(c.cache, 16, codes, a.to(BF16), v, torch.ones_like(a).to(BF16), c.slots[0])
    q = -queries(103, n or 1, group, d, BF16).abs()
    out = esb.esb_kv4_attention(q, c.cache, 16, 1, c.pages, c.lengths, starts=starts([n or 1]))
    verify_rows(c, q, out, range(n or 1))
