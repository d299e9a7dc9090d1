"""esb_rope against its definition in 64 bits.

Tolerances (fp32 work, u = 2^-24 per rounding).  A normed element: rstd one rounding (its fp64 value),
two products: 3 u.  A rotated one: each product of it with cosine or sine one more, their sum one more:
5 u of |a c| + |b s|.  6 u is allowed, then one rounding to the type."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
REL = 6 * ref.U
EPS = 1e-6


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def make(seed, *shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * torch.exp(0.5 * torch.randn(shape[-1], generator=g))).to(dtype)


def check(got, want, size):
    u, step = ref.ROUND[got.dtype], ref.STEP[got.dtype]
    off = (got.cpu().double() - want).abs()
    allowed = REL * size + u * (want.abs() + REL * size) + step
    assert bool((off <= allowed).all()), float((off / allowed).max())


SHAPES = [(1, 1, 1, 2, 2), (3, 2, 1, 7, 4), (5, 3, 1, 64, 64), (2, 4, 4, 80, 40), (17, 7, 3, 96, 48), (9, 32, 8, 128, 128),
          (4, 5, 2, 100, 96), (3, 2, 2, 129, 30), (6, 3, 1, 192, 64), (2, 2, 1, 256, 256), (3, 1, 1, 511, 128),
          (2, 3, 1, 512, 512), (300, 2, 1, 72, 72)]


@pytest.mark.parametrize("tokens,hq,hk,d,rot", SHAPES)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_heads(esb, tokens, hq, hk, d, rot, t, adjacent, norm):
    log("rope %d tokens %d|%d heads d=%d rot=%d %s adjacent=%d norm=%d" % (tokens, hq, hk, d, rot, t, adjacent, norm))
    dtype = ref.TYPES[t]
    q, k = make(d, tokens, hq, d, dtype=dtype), make(d + 1, tokens, hk, d, dtype=dtype)
    tab = ref.table(500, rot)
    pos = torch.randint(0, 500, (tokens,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    pos[0] = 499
    eps = EPS if norm else 0.0
    w = [1 + 0.3 * make(i, 1, d, dtype=torch.float32)[0] for i in (5, 6)] if norm else [None, None]
    gq, gk = esb.esb_rope(q.cuda(), k.cuda(), tab.cuda(), pos.cuda(), eps=eps, adjacent=adjacent,
                          q_w=w[0].cuda() if norm else None, k_w=w[1].cuda() if norm else None)
    for got, x, xw in ((gq, q, w[0]), (gk, k, w[1])):
        assert got.dtype == dtype
        check(got, *ref.turn(x, xw, eps, tab, pos, adjacent))
    # one of the two alone, no weights: the same code, so the same bits where the inputs are the same
    none, alone = esb.esb_rope(None, k.cuda(), tab.cuda(), pos.cuda(), eps=eps, adjacent=adjacent)
    assert none is None
    check(alone, *ref.turn(k, None, eps, tab, pos, adjacent))
    # norm only
    only, none = esb.esb_rope(q.cuda(), eps=EPS, q_w=None)
    check(only, *ref.turn(q, None, EPS, None, None, False))


@pytest.mark.parametrize("layout", ["columns", "heads first", "apart", "in place"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_pitches(esb, layout, shift):
    """Heads of fused rows, heads before tokens, at any element; nothing else is written."""
    tokens, hq, hk, d, dtype = 7, 3, 2, 80, torch.bfloat16
    tab, pos = ref.table(64, d), torch.arange(tokens, dtype=torch.int32) * 9
    q, k = make(1, tokens, hq, d, dtype=dtype), make(2, tokens, hk, d, dtype=dtype)

    def place(x):
        n = x.shape[1]
        if layout == "heads first":
            buf = torch.full((n * (tokens * d + 5) + shift,), 77.0, dtype=dtype).cuda()
            v = buf[shift:].as_strided((tokens, n, d), (d, tokens * d + 5, 1), shift)
        else:
            row = (n + 4) * (d + 3)
            buf = torch.full((tokens * row + shift,), 77.0, dtype=dtype).cuda()
            v = buf.as_strided((tokens, n, d), (row, d + (3 if layout == "apart" else 0), 1), shift)
        return buf, v

    (bq, vq), (bk, vk) = place(q), place(k)
    vq.copy_(q), vk.copy_(k)
    if layout == "in place":
        oq, ok, outs = vq, vk, (bq, bk)
    else:
        (b1, oq), (b2, ok) = place(q), place(k)
        outs = (b1, b2)
    rq, rk = esb.esb_rope(vq, vk, tab.cuda(), pos.cuda(), q_out=oq, k_out=ok, eps=EPS)
    assert rq is oq and rk is ok
    for got, x in ((oq, q), (ok, k)):
        check(got, *ref.turn(x, None, EPS, tab, pos, False))
    for buf, v, x in ((outs[0], oq, q), (outs[1], ok, k)):
        assert int((buf != 77.0).sum()) <= x.numel()
        kept = buf.clone()
        kept.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(77.0)
        assert bool((kept == 77.0).all())


def test_broadcast_input(esb):
    """A head that every token shares (pitch 0)."""
    x = make(3, 1, 2, 64, dtype=torch.float16)
    tab, pos = ref.table(50, 64), torch.arange(50, dtype=torch.int32)
    got, _ = esb.esb_rope(x.cuda().expand(50, 2, 64), None, tab.cuda(), pos.cuda())
    check(got, *ref.turn(x.expand(50, 2, 64), None, 0.0, tab, pos, False))


def test_special_values(esb):
    x = make(4, 6, 1, 64, dtype=torch.float32)
    x[1] = 0
    x[2] = 3e38                      # squares beyond fp32
    x[3, 0, 5] = float("nan")
    x[4, 0, 63] = float("inf")
    tab = ref.table(10, 32)
    pos = torch.tensor([0, 1, 0, 3, 4, 5], dtype=torch.int32)
    got, _ = esb.esb_rope(x.cuda(), None, tab.cuda(), pos.cuda(), eps=EPS)
    want, size = ref.turn(x, None, EPS, tab, pos, False)
    for i in (0, 1, 5):
        check(got[i:i + 1], want[i:i + 1], size[i:i + 1])
    # rstd of row 2 is a subnormal number of 2^-128: 21 bits
    assert bool(((got[2].cpu().double() - want[2]).abs() <= 2.0 ** -20 * size[2]).all())
    assert bool(torch.isnan(got[3]).all()) and bool(torch.isnan(got[4, 0, 63]))


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 32), (80, 40), (128, 0), (100, 96)])
def test_not_finite_stays_in_its_pair(esb, adjacent, d, rot):
    """Without a norm what is not finite reaches its own pair, and where nothing rotates itself only."""
    x = make(9, 3, 2, d, dtype=torch.bfloat16)
    tab, pos = ref.table(9, rot), torch.tensor([0, 5, 8], dtype=torch.int32)
    how = dict(table=tab.cuda(), positions=pos.cuda()) if rot else {}
    clean, _ = esb.esb_rope(x.cuda(), None, adjacent=adjacent, **how)
    for at in {0, rot // 2, max(rot - 1, 0), rot, d - 1} - {d}:
        y = x.clone()
        y[1, 1, at] = float("inf")
        got, _ = esb.esb_rope(y.cuda(), None, adjacent=adjacent, **how)
        pair = {at}
        if at < rot:
            pair = {at, at ^ 1} if adjacent else {at, (at + rot // 2) % rot}
        keep = torch.ones_like(got, dtype=torch.bool)
        keep[1, 1, list(pair)] = False
        assert torch.equal(got[keep], clean[keep])
        assert not bool(torch.isfinite(got[1, 1, list(pair)]).any())


def test_positions_outside_the_table(esb):
    x = make(5, 5, 3, 96, dtype=torch.bfloat16)
    tab = ref.table(20, 64)
    pos = torch.tensor([0, -1, 19, 20, 2 ** 31 - 1], dtype=torch.int32)
    got, _ = esb.esb_rope(x.cuda(), None, tab.cuda(), pos.cuda())
    want, size = ref.turn(x, None, 0.0, tab, pos.clamp(0, 19), False)
    for i in (0, 2):
        check(got[i:i + 1], want[i:i + 1], size[i:i + 1])
    for i in (1, 3, 4):
        assert bool(torch.isnan(got[i]).all())


def test_nothing_to_do(esb):
    z = torch.zeros(0, 3, 64, dtype=torch.bfloat16, device="cuda")
    q, k = esb.esb_rope(z, z, ref.table(4, 64).cuda(), torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert q.shape == k.shape == z.shape


def test_binding_refusals(esb):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    tab, pos = ref.table(8, 64).cuda(), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(positions=pos[:3]), dict(table=tab[:, :62]), dict(table=None), dict(k=x[:3]), dict(k=x[..., :32]),
                dict(k=x.half()), dict(q_out=x[:, :1]), dict(q=x[0]), dict(q=x.transpose(1, 2))):
        with pytest.raises(ValueError):
            esb.esb_rope(**{**dict(q=x, table=tab, positions=pos), **bad})
    for bad in (dict(positions=pos.long()), dict(table=tab.double()), dict(positions=None), dict(q=x.double()),
                dict(q_w=tab[0].double(), eps=1e-5), dict(positions=pos.cpu())):
        with pytest.raises(TypeError):
            esb.esb_rope(**{**dict(q=x, table=tab, positions=pos), **bad})
    with pytest.raises(esb.EsbError):
        esb.esb_rope(x, None, tab, pos, q_w=tab[0])          # weights without a norm


def test_streams(esb):
    """On a stream given as an object or a handle, behind the work that makes its input."""
    x = make(6, 400, 8, 128, dtype=torch.bfloat16).cuda()
    tab, pos = ref.table(400, 128).cuda(), torch.arange(400, dtype=torch.int32).cuda()
    want, _ = esb.esb_rope(x, None, tab, pos, eps=EPS)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for given in (s, s.cuda_stream):
        with torch.cuda.stream(s):
            y = x.float().mul(1).to(torch.bfloat16)
        got, _ = esb.esb_rope(y, None, tab, pos, eps=EPS, stream=given)
        s.synchronize()
        assert torch.equal(got, want)
