"""The 4-bit cache: appending, packing and reading back.

Appended keys are computed in fp64 (a few 2^-53 from the exact value) and rounded to fp32 before they get
their codes, as the definition says: a code differs only where a value lies within that of a border of
two fp32 numbers, about one in 2^28 elements; values, scales and codes are compared for equality."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
EPS = 1e-6
CODE_OF_LEVEL = torch.tensor([6, 7, 0, 1, 2, 3, 4, 5], dtype=torch.uint8)      # ESB(4,1) codes of 0, .5, 1, ..


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def make(seed, *shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * torch.exp(0.7 * torch.randn(shape[-1], generator=g))).to(dtype)


def new_cache(esb, pages, page, heads, d, fill=0xA5):
    return torch.full((pages, esb.esb_kv4_page_size(page, heads, d)), fill, dtype=torch.uint8, device="cuda")


def same(got, want):
    got, want = got.cpu().double(), want.double()
    assert bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())


@pytest.mark.parametrize("heads,d,page,tokens", [(1, 32, 16, 1), (2, 64, 16, 37), (3, 96, 32, 50), (8, 128, 64, 200),
                                                 (1, 160, 16, 33), (2, 192, 128, 130), (2, 224, 16, 17),
                                                 (2, 256, 16, 70)])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("how", ["plain", "halves", "adjacent"])
def test_append(esb, heads, d, page, tokens, t, how):
    log("append heads=%d d=%d page=%d tokens=%d %s %s" % (heads, d, page, tokens, t, how))
    dtype = ref.TYPES[t]
    g = torch.Generator().manual_seed(d)
    k, v = make(1, tokens, heads, d, dtype=dtype), make(2, tokens, heads, d, dtype=dtype)
    pages = tokens // page + 2
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    rot = 0 if how == "plain" else d if how == "halves" else d // 2
    tab = ref.table(300, rot) if rot else None
    pos = torch.randint(0, 300, (tokens,), generator=g, dtype=torch.int32) if rot else None
    eps, w = (EPS, 1 + 0.2 * torch.randn(d, generator=g)) if how == "halves" else (0.0, None)
    q = make(3, tokens, 2 * heads, d, dtype=dtype) if how == "adjacent" else None
    cache = new_cache(esb, pages, page, heads, d)
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    out = esb.esb_kv4_append(cache, page, dev(k), dev(v), dev(slots), dev(tab), dev(pos), k_w=dev(w), eps=eps,
                             adjacent=how == "adjacent", q=dev(q))
    gk, gka, gv, gva = esb.esb_kv4_unpack(cache, page, heads, d, slots.cuda())
    y, _ = ref.turn(k, w, eps, tab, pos, how == "adjacent")
    for got, ga, exact in ((gk, gka, y.float()), (gv, gva, v.float())):
        values, alpha = ref.codes(exact)
        same(ga, alpha)
        same(got, values)
    if q is None:
        assert out is None
    else:
        want, size = ref.turn(q, None, 0.0, tab, pos, True)
        off = (out.cpu().double() - want).abs()
        assert bool((off <= 2 * ref.U * size + ref.ROUND[dtype] * want.abs() * (1 + ref.U) + ref.STEP[dtype]).all())
    # no other slot was touched: every other token's codes and scales are those of the fill
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots] = False
    rest = rest.nonzero()[:, 0].cuda()
    before = esb.esb_kv4_unpack(new_cache(esb, pages, page, heads, d), page, heads, d, rest)
    for a, b in zip(esb.esb_kv4_unpack(cache, page, heads, d, rest), before):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_append_special(esb):
    """Zeros, ties, NaN, infinities, the largest and smallest numbers; a group by itself."""
    d, page = 64, 16
    k = torch.zeros(9, 1, d)
    k[1, 0, :32] = torch.tensor([6.0] + [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25] * 3 + [0.2499, -0.74] * 3 + [-6.0])
    k[2, 0, 3] = float("nan")
    k[3, 0, 40] = float("inf")
    k[4, 0] = 3.4e38
    k[5, 0] = 1e-45
    k[6, 0, 0] = -1e-38
    k[7, 0, 10] = 2.0 ** -126
    k[8, 0] = -0.0
    cache = new_cache(esb, 1, page, 1, d)
    slots = torch.arange(9)
    esb.esb_kv4_append(cache, page, k.cuda(), (-k).cuda(), slots.cuda())
    gk, gka, gv, gva = esb.esb_kv4_unpack(cache, page, 1, d, slots.cuda())
    for got, ga, x in ((gk, gka, k), (gv, gva, -k)):
        values, alpha = ref.codes(x)
        same(ga, alpha)
        same(got, values)
        assert not bool(torch.signbit(got.float()[got.float() == 0]).any())


def test_slots_outside(esb):
    """Tokens without a slot in the cache are passed over; reading such slots gives zeros under NaN."""
    heads, d, page, pages = 2, 64, 32, 3
    k = make(5, 6, heads, d, dtype=torch.bfloat16)
    slots = torch.tensor([-1, 95, 96, 0, -2 ** 62, 2 ** 62])
    cache = new_cache(esb, pages, page, heads, d)
    guard = cache.clone()
    q = esb.esb_kv4_append(cache, page, k.cuda(), k.cuda(), slots.cuda(), q=k.cuda())
    assert torch.equal(q.cpu(), k)
    values, alpha = ref.codes(k.float())
    gk, gka, gv, gva = esb.esb_kv4_unpack(cache, page, heads, d, slots.cuda())
    for i in (1, 3):
        same(gk[i], values[i]), same(gka[i], alpha[i]), same(gv[i], values[i]), same(gva[i], alpha[i])
    for i in (0, 2, 4, 5):
        assert not bool(gk[i].float().any()) and not bool(gv[i].float().any())
        assert bool(torch.isnan(gka[i]).all()) and bool(torch.isnan(gva[i]).all())
    assert torch.equal(cache[1], guard[1])


@pytest.mark.parametrize("heads,d,page", [(1, 32, 16), (3, 96, 32), (2, 256, 64)])
def test_pack(esb, heads, d, page):
    g = torch.Generator().manual_seed(7)
    n = 3 * page
    codes = torch.randint(0, 256, (2, n, heads, d), generator=g, dtype=torch.uint8)
    alpha = torch.randn(2, n, heads, d // 32, generator=g).to(torch.bfloat16)
    slots = torch.randperm(n, generator=g)
    cache = new_cache(esb, 3, page, heads, d)
    esb.esb_kv4_pack(cache, page, codes[0].cuda(), alpha[0].cuda(), codes[1].cuda(), alpha[1].cuda(), slots.cuda())
    k, ka, v, va = esb.esb_kv4_unpack(cache, page, heads, d, slots.cuda())
    from decoder_ref import CODE_VALUES
    for got, ga, c, a in ((k, ka, codes[0], alpha[0]), (v, va, codes[1], alpha[1])):
        assert torch.equal(got.cpu().double(), CODE_VALUES[(c & 15).long()])
        assert torch.equal(ga.cpu(), a)


def test_layout(esb):
    """The documented places of codes and scales in a page."""
    heads, d, page = 2, 96, 16
    G = d // 32
    k, v = make(8, page, heads, d, dtype=torch.float32), make(9, page, heads, d, dtype=torch.float32)
    cache = new_cache(esb, 2, page, heads, d)
    esb.esb_kv4_append(cache, page, k.cuda(), v.cuda(), torch.arange(page, 2 * page).cuda())
    blocks = cache[1].cpu().reshape(heads, 36 * G * page)

    def nibbles(x):
        values, alpha = ref.codes(x)
        m = torch.searchsorted(ref.LEVELS, values.abs().contiguous()).to(torch.uint8)
        return m | ((values < 0).to(torch.uint8) << 3), alpha

    for h in range(heads):
        b = blocks[h]
        kn, ka = nibbles(k[:, h:h + 1])
        vn, va = nibbles(v[:, h:h + 1])
        words = kn[:, 0].reshape(page, G, 4, 8).transpose(1, 2)            # [token][a][g][8]
        assert torch.equal(b[:16 * G * page].reshape(page, 4, G, 4), words[..., 0::2] | words[..., 1::2] << 4)
        pairs = vn[:, 0].reshape(page // 4, 4, G, 16, 2).permute(0, 3, 2, 1, 4)   # [run][a][g][token][2]
        assert torch.equal(b[16 * G * page:32 * G * page].reshape(page // 4, 16, G, 4),
                           pairs[..., 0] | pairs[..., 1] << 4)
        for at, a in ((32, ka), (34, va)):
            s = b[at * G * page:(at + 2) * G * page].contiguous().view(torch.bfloat16).reshape(page // 4, G, 4)
            assert torch.equal(s, a[:, 0].reshape(page // 4, 4, G).transpose(1, 2))


def test_strided_columns(esb):
    """Keys and values as columns of one product's rows, at odd elements."""
    heads, d, page, n = 3, 64, 16, 21
    buf = make(10, n, 2 * heads * d + 7, dtype=torch.float16).cuda()
    k = buf[:, 1:1 + heads * d].unflatten(1, (heads, d))
    v = buf[:, 3 + heads * d:3 + 2 * heads * d].unflatten(1, (heads, d))
    slots = torch.arange(n).cuda()
    a, b = new_cache(esb, 2, page, heads, d), new_cache(esb, 2, page, heads, d)
    esb.esb_kv4_append(a, page, k, v, slots)
    esb.esb_kv4_append(b, page, k.contiguous(), v.contiguous(), slots)
    assert torch.equal(a, b)


def test_far_slots(esb):
    """Offsets beyond 2^32 bytes."""
    heads, d, page = 8, 128, 4096
    size = esb.esb_kv4_page_size(page, heads, d)
    pages = 2 ** 32 // size + 3
    cache = torch.empty(pages, size, dtype=torch.uint8, device="cuda")
    cache[-1].zero_(), cache[0].zero_()
    k = make(11, 5, heads, d, dtype=torch.bfloat16)
    slots = torch.arange(pages * page - 5, pages * page).cuda()
    esb.esb_kv4_append(cache, page, k.cuda(), k.cuda(), slots)
    got = esb.esb_kv4_unpack(cache, page, heads, d, slots)
    values, alpha = ref.codes(k.float())
    same(got[0], values), same(got[1], alpha), same(got[2], values), same(got[3], alpha)
    assert not bool(cache[0].any())


def test_binding_refusals(esb):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache, slots = new_cache(esb, 2, 16, 2, 64), torch.arange(4).cuda()
    for bad in (dict(cache=cache[:, :-1]), dict(cache=cache[0]), dict(cache=cache.float()), dict(page=32), dict(v=x[:3]),
                dict(v=x.half()), dict(slots=slots[:3]), dict(k=x[0]), dict(q=x[:2])):
        with pytest.raises(ValueError):
            esb.esb_kv4_append(**{**dict(cache=cache, page=16, k=x, v=x, slots=slots), **bad})
    for page, d in ((24, 64), (8, 64), (16, 48)):      # shapes that the library does not take
        y = x[..., :d]
        with pytest.raises(esb.EsbError):
            esb.esb_kv4_append(cache.new_zeros(2, 2 * page * 36 * (d // 32)), page, y, y, slots)
    with pytest.raises(TypeError):
        esb.esb_kv4_append(cache, 16, x, x, slots.int())
    with pytest.raises(TypeError):
        esb.esb_kv4_append(cache, 16, x.double(), x.double(), slots)
    with pytest.raises(TypeError):
        esb.esb_kv4_unpack(cache, 16, 2, 64, None)
