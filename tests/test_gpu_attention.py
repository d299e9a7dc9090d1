"""esb_attention against its definition in 64 bits.

Tolerances: attention_ref.check, from the roundings that the operator makes: fp32 scores and sums, one
rounding of each probability to the inputs' type, one of the output."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def make(seed, *shape, dtype, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


def starts(counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


def verify(q, k, v, out, nq, nk, causal, scale=None):
    a = b = 0
    d = q.shape[2]
    for n, m in zip(nq, nk):
        if n:
            last = torch.arange(n) + m - n if causal else torch.full((n,), m - 1)
            want = ref.attend(q[a:a + n], k[b:b + m], v[b:b + m], last, d ** -0.5 if scale is None else scale)
            ref.check(out[a:a + n], *want, keys=m, d=d, p_round=ref.ROUND[q.dtype],
                      p_step=2.0 ** -25 if q.dtype == torch.float16 else 0.0)
            if causal:
                assert not bool(out[a:a + max(0, min(n, n - m))].any())
        a, b = a + n, b + m


PACKS = [([1], [1]), ([1, 0, 2, 33], [1, 0, 2, 33]), ([64, 65, 63], [64, 65, 63]), ([130, 1, 127, 200], [130, 1, 127, 200]),
         ([5, 1, 0, 40], [300, 77, 12, 129]), ([9, 70, 3], [4, 0, 3])]


@pytest.mark.parametrize("nq,nk", PACKS)
@pytest.mark.parametrize("kv,group,d", [(1, 1, 8), (2, 3, 64), (1, 8, 80), (3, 1, 96), (2, 4, 128), (1, 5, 136), (2, 2, 192),
                                        (1, 3, 256)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_packs(esb, nq, nk, kv, group, d, causal, t):
    log("attention nq=%s nk=%s kv=%d group=%d d=%d causal=%d %s" % (nq, nk, kv, group, d, causal, t))
    dtype = ref.TYPES[t]
    q = make(1, sum(nq) + 2, kv * group, d, dtype=dtype)
    k, v = (make(s, sum(nk) + 1, kv, d, dtype=dtype) for s in (2, 3))
    out = torch.full_like(q, 9.0)
    got = esb.esb_attention(q, k, v, starts(nq), starts(nk), causal=causal, out=out)
    assert got is out
    verify(q, k, v, out, nq, nk, causal)
    assert bool((out[sum(nq):] == 9.0).all())          # rows behind the last sequence


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv,group,d,n", [(2, 4, 128, 1500), (1, 3, 64, 2049), (1, 2, 256, 1100)])
def test_long(esb, t, kv, group, d, n):
    log("attention long %s d=%d n=%d" % (t, d, n))
    dtype = ref.TYPES[t]
    q = make(4, n, kv * group, d, dtype=dtype)
    k, v = (make(s, n, kv, d, dtype=dtype) for s in (5, 6))
    out = esb.esb_attention(q, k, v, starts([n]))
    verify(q, k, v, out, [n], [n], True)
    assert torch.equal(out, esb.esb_attention(q, k, v, starts([n])))


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_sharp_and_growing_scores(esb, t):
    n, d = 700, 128
    dtype = ref.TYPES[t]
    q, k, v = make(7, n, 2, d, dtype=dtype, size=6.0), make(8, n, 1, d, dtype=dtype, size=4.0), make(9, n, 1, d, dtype=dtype)
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n]), scale=0.5), [n], [n], True, scale=0.5)
    k = (k.float().abs() * (torch.arange(n, device="cuda")[:, None, None] / 40).floor()).to(dtype)
    q = (q.float().abs() / 60).to(dtype)
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n]), causal=False), [n], [n], False)
    verify(q, -k, v, esb.esb_attention(q, -k, v, starts([n])), [n], [n], True)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("d,at", [(64, 70), (128, 0), (128, 130), (256, 40)])
def test_not_finite(esb, value, what, d, at):
    """What is not finite reaches the queries that see it and no others."""
    nq = [150, 60]
    q, k, v = (make(s, 210, 2 if s == 10 else 1, d, dtype=torch.bfloat16) for s in (10, 11, 12))
    clean = esb.esb_attention(q, k, v, starts(nq))
    x = k if what == "k" else v
    x[at, 0, 5] = value
    out = esb.esb_attention(q, k, v, starts(nq))
    assert torch.equal(out[:at], clean[:at]) and torch.equal(out[150:], clean[150:])
    if what == "v":
        want = torch.full_like(out[at:150, :, 5], value)
        assert torch.equal(torch.isnan(out[at:150, :, 5]), torch.isnan(want))
        assert bool(((out[at:150, :, 5] == want) | torch.isnan(want)).all())
        rest = [i for i in range(d) if i != 5]
        assert torch.equal(out[:, :, rest], clean[:, :, rest])
    else:
        # scores of NaN or +infinity make a row NaN, of -infinity drop out
        o = ref.attend(q[:150].cpu(), k[:150].cpu(), v[:150].cpu(), torch.arange(150), d ** -0.5)[0]
        assert torch.equal(torch.isnan(out[:150].cpu()), torch.isnan(o))
    q[3] = float("nan")
    out2 = esb.esb_attention(q, k, v, starts(nq))
    assert bool(torch.isnan(out2[3]).all()) and torch.equal(out2[4:].isnan(), out[4:].isnan())


def test_neighbours_in_the_pack(esb):
    """A sequence of NaN between others reaches none of them."""
    n = [40, 30, 50]
    q, k, v = (make(s, 120, 2, 64, dtype=torch.float16) for s in (13, 14, 15))
    clean = esb.esb_attention(q, k, v, starts(n), causal=False)
    for x in (k, v):
        x[40:70] = float("nan")
    out = esb.esb_attention(q, k, v, starts(n), causal=False)
    assert torch.equal(out[:40], clean[:40]) and torch.equal(out[70:], clean[70:])
    assert bool(torch.isnan(out[40:70]).all())


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_pitches(esb, shift):
    """Columns of fused rows at any element, heads before tokens; nothing else is written."""
    n, hq, hk, d = 90, 6, 2, 80
    row = (hq + 2 * hk) * d + 5
    buf = make(16, n * row + 8, dtype=torch.bfloat16)
    f = [buf.as_strided((n, h, d), (row, d, 1), shift + at * d) for h, at in ((hq, 0), (hk, hq), (hk, hq + hk))]
    want = esb.esb_attention(*(x.contiguous() for x in f), starts([70, 20]))
    ob = torch.full((hq * (n * d + 3) + 8,), 2.0, dtype=torch.bfloat16, device="cuda")
    o = ob.as_strided((n, hq, d), (d, n * d + 3, 1), shift)
    esb.esb_attention(*f, starts([70, 20]), out=o)
    assert torch.equal(o, want)
    o.fill_(2.0)
    assert bool((ob == 2.0).all())


def test_starts_of_anything(esb):
    q, k, v = (make(s, 60, 2, 64, dtype=torch.bfloat16) for s in (17, 18, 19))
    buf = torch.full((80, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    for s in ([0, -5, 70, 7], [60, 30, 2, 0], [2 ** 31 - 1, 0, 9, 2 ** 31 - 1], [-2 ** 31, 20, 10, 60]):
        for ks in (None, [5, 2 ** 31 - 1, -9, 30]):
            ks = None if ks is None else torch.tensor(ks, dtype=torch.int32, device="cuda")
            esb.esb_attention(q, k, v, torch.tensor(s, dtype=torch.int32, device="cuda"), ks, out=buf[10:70])
            assert bool((buf[:10] == 3.0).all()) and bool((buf[70:] == 3.0).all())


def test_many_sequences(esb):
    n = [(7 * i) % 11 for i in range(200)]
    q, k, v = (make(s, sum(n), 4 if s == 20 else 2, 64, dtype=torch.float16) for s in (20, 21, 22))
    verify(q, k, v, esb.esb_attention(q, k, v, starts(n)), n, n, True)


def test_nothing_to_do(esb):
    z = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert esb.esb_attention(z, z, z, starts([])).shape == z.shape
    # queries without a key at all
    q = make(23, 5, 2, 64, dtype=torch.bfloat16)
    assert not bool(esb.esb_attention(q, z, z, starts([5]), starts([0])).any())


def test_graph_and_stream(esb):
    n = [300, 41]
    xs = [[make(s + i, 341, 2, 128, dtype=torch.bfloat16) for i in range(3)] for s in (24, 27, 30)]
    st = starts(n)
    want = [esb.esb_attention(*x, st) for x in xs]
    ins = [x.clone() for x in xs[0]]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = esb.esb_attention(*ins, st)
    for x, w in zip(xs + xs, want + want):
        for a, b in zip(ins, x):
            a.copy_(b)
        g.replay()
        assert torch.equal(out, w)
        torch.cuda.synchronize()
        assert torch.equal(esb.esb_attention(*x, st), w)
    s = torch.cuda.Stream()
    for given in (s, s.cuda_stream):
        with torch.cuda.stream(s):
            y = [x.float().to(torch.bfloat16) for x in xs[1]]
        got = esb.esb_attention(*y, st, stream=given)
        s.synchronize()
        assert torch.equal(got, want[1])


def test_binding_refusals(esb):
    q, k = make(33, 9, 4, 64, dtype=torch.bfloat16), make(34, 9, 2, 64, dtype=torch.bfloat16)
    st = starts([9])
    call = dict(q=q, k=k, v=k, q_starts=st)
    for bad in (dict(k=k[..., :32]), dict(v=k[:8]), dict(v=k[:, :1]), dict(k=k.half()), dict(q_starts=st[:0]),
                dict(k_starts=starts([3, 6])), dict(out=q[:8]), dict(q=q[0])):
        with pytest.raises(ValueError):
            esb.esb_attention(**{**call, **bad})
    for bad in (dict(q_starts=st.long()), dict(q_starts=st.cpu()), dict(q_starts=None), dict(q=q.double())):
        with pytest.raises(TypeError):
            esb.esb_attention(**{**call, **bad})
    for bad in (dict(q=q[:, :3]), dict(q=q.float(), k=k.float(), v=k.float()), dict(out=q), dict(scale=-1.0),
                dict(k=k[:8], v=k[:8])):
        with pytest.raises(esb.EsbError):
            esb.esb_attention(**{**call, **bad})
