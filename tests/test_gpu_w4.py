"""Group-scaled 4-bit weights: quantization, packing, unpacking, against the definition in 64 bits.
The candidates' scales are fp32 operations rounded to bf16 and the codes exact nearest values, so
scales and codes are equal, not close, except where two candidates' errors agree to fp64 rounding."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def weights(seed, N, K, t):
    g = torch.Generator().manual_seed(seed)
    w = 0.05 * torch.randn(N, K, generator=g) * torch.exp(torch.randn(N, 1, generator=g))
    return w.to(ref.TYPES[t])


def factors(n):
    return [1 - j / 32 for j in range(n)]


@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (5, 31), (33, 32), (40, 65), (64, 1000),
                                 (100, 257), (15, 2047)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_quantize(esb, N, K, group, t):
    log("w4 quantize N=%d K=%d group=%d %s" % (N, K, group, t))
    w = weights(N + K, N, K, t)
    for n in (1, 5, 16):
        f = None if n == 1 else torch.tensor(factors(n)).cuda()
        w4 = esb.esb_w4_quantize(w.cuda(), group, f)
        assert w4.numel() == esb.esb_w4_size(N, K, group)
        q, alpha = esb.esb_w4_unpack(w4, N, K, group)
        rq, ra = ref.quantize(w, group, factors(n))
        assert torch.equal(alpha.cpu().double(), ra)
        assert torch.equal(q.cpu().double(), rq)


def test_ties_go_to_the_larger_magnitude(esb):
    # alpha = 1 exactly (the largest weight is 6): midpoints, their neighbours, zeros of both signs
    mids = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    up = np.nextafter(np.float32(mids), np.float32(9))
    down = np.nextafter(np.float32(mids), np.float32(0))
    row = np.concatenate([mids, up, down, [6.0, 0.0, -0.0]]).astype(np.float32)
    w = torch.from_numpy(np.stack([row, -row]))
    q, alpha = esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), 32), 2, row.size, 32)
    assert alpha.cpu().flatten().tolist() == [1.0, 1.0]
    want = [.5, 1, 1.5, 2, 3, 4, 6] * 2 + [0, .5, 1, 1.5, 2, 3, 4] + [6, 0, 0]
    assert q.cpu().float()[0].tolist() == want
    assert q.cpu().float()[1].tolist() == [-v if v else 0 for v in want]
    assert not bool(torch.signbit(q.cpu().float()[0, -2:]).any())


def test_candidates_that_tie(esb):
    """Equal errors under different scales: the lowest index, among two, three or all candidates, also
    where fp32 sums cannot tell them apart."""
    w = torch.zeros(40, 64)
    w[:, 0] = 6.0                       # exact under alpha = 1, 2 and 4
    w[1, :32] = 6.0
    w[2, 40] = 6.0 * 2.0 ** -100
    w[3] = 0
    w[4:, 1] = torch.linspace(-6, 6, 36)
    for f in ([0.5, 1.0, 2.0], [0.5, 2.0, 1.0], [4.0, 2.0, 1.0, 0.5], [0.5, 1.0, 1.0, 1.0 + 2.0 ** -20], [2.0] * 9):
        q, alpha = esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), 32, torch.tensor(f).cuda()), 40, 64, 32)
        rq, ra = ref.quantize(w, 32, f)
        assert torch.equal(alpha.cpu().double(), ra), f
        assert torch.equal(q.cpu().double(), rq), f


@pytest.mark.parametrize("scale", [2.0 ** -60, 1.0, 2.0 ** 90])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_any_size_of_weights(esb, scale, t):
    """Weights whose squares leave fp32, and factors far from 1 (64 of them)."""
    w = (weights(11, 50, 300, "f32") * scale).to(ref.TYPES[t])
    w[:, ::7] = 0
    f = [2.0 ** e for e in range(-34, -2)] + [1 - j / 64 for j in range(32)]
    q, alpha = esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), 64, torch.tensor(f).cuda()), 50, 300, 64)
    rq, ra = ref.quantize(w, 64, f)
    assert torch.equal(alpha.cpu().double(), ra)
    assert torch.equal(q.cpu().double(), rq)
    only = [2.0 ** -120]                # every weight far above its scale
    w4 = esb.esb_w4_quantize(w.cuda(), 64, torch.tensor(only).cuda())
    assert not bool(w4[:1024 * 10].view(2, 5, 1024)[1, 4].view(64, 16)[18:32].any())     # rows past 50
    q, alpha = esb.esb_w4_unpack(w4, 50, 300, 64)
    rq, ra = ref.quantize(w, 64, only)
    assert torch.equal(alpha.cpu().double(), ra)
    assert torch.equal(q.cpu().double(), rq)


def test_groups_without_a_scale(esb):
    """Zeros, NaN, infinities, the largest and the smallest weights; factors that are passed over."""
    inf, nan = float("inf"), float("nan")
    w = weights(7, 8, 96, "f32")
    w[0, :32] = 0
    w[1, 40] = nan
    w[2, 95] = -inf
    w[3, :32] = 3e38
    w[4, :32] = 1e-42
    f = torch.tensor([nan, -1.0, 0.0, inf, 2.0, 1.0, 0.5])
    q, alpha = [v.cpu() for v in esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), 32, f.cuda()), 8, 96, 32)]
    assert float(alpha[0, 0]) == 2.0 ** -126 and not bool(q[0, :32].float().any())
    for n, g in ((1, 1), (2, 2)):
        assert bool(torch.isnan(alpha[n, g])) and not bool(q[n, 32 * g:32 * g + 32].float().any())
    assert int(torch.isnan(alpha.float()).sum()) == 2
    assert float(alpha[4, 0]) == 2.0 ** -126 and not bool(q[4, :32].float().any())
    clean = torch.nan_to_num(w, nan=0.0, posinf=0.0, neginf=0.0)
    rq, ra = ref.quantize(clean, 32, [2.0, 1.0, 0.5])     # 2 * 3e38 overflows: passed over
    ok = torch.isfinite(alpha.float())
    assert torch.equal(alpha.double()[ok], ra[ok])
    okk = ok.repeat_interleave(32, 1)
    assert torch.equal(q.double()[okk], rq[okk])
    only = torch.tensor([nan, -1.0])
    q, alpha = esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), 32, only.cuda()), 8, 96, 32)
    assert bool(torch.isnan(alpha.float()).all()) and not bool(q.float().any())


@pytest.mark.parametrize("N,K,group", [(16, 128, 128), (18, 200, 32), (1, 1, 64), (50, 999, 128), (33, 4096, 64)])
def test_pack_layout_and_unpack(esb, N, K, group):
    """Every code and scale stands where the header says; unpack returns them."""
    rng = np.random.default_rng(N + K)
    codes = torch.from_numpy(rng.integers(0, 256, (N, K + 3), dtype=np.uint8))   # bits above 3 ignored
    groups = -(-K // group)
    alpha = torch.from_numpy(rng.standard_normal((N, groups)).astype(np.float32)).to(torch.bfloat16)
    w4 = esb.esb_w4_pack(codes.cuda()[:, 3:], alpha.cuda(), group)
    want = ref.CODE_VALUES[(codes[:, 3:] & 15).long()]
    q, a = esb.esb_w4_unpack(w4, N, K, group)
    assert torch.equal(q.cpu().double(), want) and torch.equal(a.cpu(), alpha)
    assert not bool(torch.signbit(q.cpu().float()[q.cpu().float() == 0]).any())
    raw = w4.cpu().numpy()
    tiles, chunks = -(-N // 32), -(-K // 64)
    per_row = -(-64 * chunks // group)
    assert raw.size == 1024 * tiles * chunks + 64 * tiles * per_row
    words = raw[:1024 * tiles * chunks].view(np.uint32)
    n, k = np.meshgrid(np.arange(32 * tiles), np.arange(64 * chunks), indexing="ij")
    c = k % 64
    at = 256 * ((n // 32) * chunks + k // 64) + 4 * (32 * ((c // 16) % 2) + n % 32) + c // 32 + 2 * ((c // 8) % 2)
    nib = (words[at] >> (4 * (c % 8)).astype(np.uint32)) & 15
    val = ref.LEVELS.numpy()[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    np.testing.assert_array_equal(val[:N, :K], want.numpy())
    assert not nib[N:].any() and not nib[:, K:].any()
    sc = torch.from_numpy(raw[1024 * tiles * chunks:].copy()).view(torch.bfloat16).view(tiles, per_row, 32)
    sc = sc.permute(0, 2, 1).reshape(32 * tiles, per_row)
    assert torch.equal(sc[:N, :groups], alpha)
    assert not bool(sc[N:].any()) and not bool(sc[:, groups:].any())


def test_pitched_inputs_and_outputs(esb):
    w = weights(3, 21, 333, "bf16")
    big = torch.full((21, 345), float("nan"), dtype=torch.bfloat16)
    big[:, 5:338] = w
    f = torch.tensor(factors(4)).cuda()
    a = esb.esb_w4_quantize(w.cuda(), 64, f)
    b = esb.esb_w4_quantize(big.cuda()[:, 5:338], 64, f)
    assert torch.equal(a, b)
    values = torch.full((21, 340), 7.0, device="cuda").to(torch.float8_e4m3fn)
    alpha = torch.full((21, 9), 7.0, device="cuda", dtype=torch.bfloat16)
    esb.esb_w4_unpack(a, 21, 333, 64, values=values[:, 3:336], alpha=alpha[:, 1:7])
    q, al = esb.esb_w4_unpack(a, 21, 333, 64)
    assert torch.equal(values[:, 3:336].float(), q.float()) and torch.equal(alpha[:, 1:7], al)
    assert bool((values[:, :3].float() == 7).all()) and bool((values[:, 336:].float() == 7).all())
    assert bool((alpha[:, :1] == 7).all()) and bool((alpha[:, 7:] == 7).all())


def test_codes_of_the_projection(esb):
    """A matrix projected with one scale per tensor packs to the same codes as its groups."""
    w = weights(5, 32, 256, "f32").cuda()
    alpha = torch.tensor([0.03125], device="cuda")
    codes = esb.esb_project(w, alpha, 4, 2)
    w4 = esb.esb_w4_pack(codes, torch.full((32, 2), 0.03125, device="cuda", dtype=torch.bfloat16), 128)
    q, a = esb.esb_w4_unpack(w4, 32, 256, 128)
    assert torch.equal(q.float() * 0.03125, esb.esb_dequantize(codes, alpha, 4, 2))


def test_refusals(esb):
    w = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    for group in (0, 16, 48, 256):
        assert esb.esb_w4_size(32, 64, group) == 0
        with pytest.raises(esb.EsbError):
            esb.esb_w4_quantize(w, group)
    with pytest.raises(esb.EsbError):
        esb.esb_w4_quantize(w, 32, torch.ones(65, device="cuda"))
    with pytest.raises(esb.EsbError):
        esb.esb_w4_quantize(w, 32, w4=torch.empty(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(esb.EsbError):
        esb.esb_w4_unpack(torch.empty(100, dtype=torch.uint8, device="cuda"), 32, 64, 32)
    with pytest.raises(TypeError):
        esb.esb_w4_quantize(w.double(), 32)
    with pytest.raises(TypeError):
        esb.esb_w4_pack(w, w, 32)
    with pytest.raises(ValueError):
        esb.esb_w4_pack(torch.zeros(32, 64, dtype=torch.uint8, device="cuda"), w, 32)
    assert esb.esb_w4_quantize(torch.zeros(0, 64, device="cuda"), 32).numel() <= 1


def near_groups(f1):
    """Rows of 32 fp32 weights whose candidates 1 and f1 differ by a part in 10^6 or less, the first's error
    the smaller one and nearly all of it one weight's next to a cell bound: (top, that weight, one more)."""
    levels = ref.LEVELS.numpy()
    mids = (levels[1:] + levels[:-1]) / 2

    def squares(a, w):
        return (w - a * levels[np.searchsorted(mids, w / a, side="right")]) ** 2

    rows = []
    for man in range(0, 128, 8):
        a0 = 1 + man / 128
        top = np.float32(6 * a0)
        a1 = float(torch.tensor(float(np.float32(top * np.float32(f1)) / np.float32(6))).to(torch.bfloat16))
        for mid in (5.0, 3.5, 2.5, 1.75):
            for k in (-2, -1, 1, 2):
                s = np.float32(mid * a0)
                for _ in range(abs(k)):
                    s = np.nextafter(s, np.float32(100 if k > 0 else 0))
                two = np.array([top, s], dtype=np.float64)

                def ratio(u):
                    return ((squares(a1, two).sum() + squares(a1, u)) / (squares(a0, two).sum() + squares(a0, u))) - 1

                u = np.linspace(0, 6 * a0, 1001)
                f = ratio(u) - 4e-7
                for i in np.nonzero(np.sign(f[1:]) != np.sign(f[:-1]))[0][:3]:
                    lo, hi = u[i], u[i + 1]
                    for _ in range(40):
                        m = (lo + hi) / 2
                        if np.sign(ratio(np.array([m]))[0] - 4e-7) == np.sign(f[i]):
                            lo = m
                        else:
                            hi = m
                    near = (np.float32(lo).view(np.uint32).astype(np.int64) + np.arange(-4, 5)).clip(0)
                    near = near.astype(np.uint32).view(np.float32)
                    off = ratio(near.astype(np.float64))
                    rows += [(top, s, v) for v in near[(off > 1e-9) & (off < 1.5e-6)][:3]]
    w = torch.zeros(len(rows), 32)
    w[:, :3] = torch.tensor(rows)
    return w


@pytest.mark.parametrize("f1", [31 / 32, 0.9, 1.03])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_candidates_a_part_in_a_million_apart(esb, f1, group):
    w = torch.nn.functional.pad(near_groups(f1), (0, group - 32))
    assert w.shape[0] > 500
    q, alpha = esb.esb_w4_unpack(esb.esb_w4_quantize(w.cuda(), group, torch.tensor([1.0, f1]).cuda()),
                                 w.shape[0], group, group)
    rq, ra = ref.quantize(w, group, [1.0, f1])
    assert torch.equal(alpha.cpu().double(), ra)
    assert torch.equal(q.cpu().double(), rq)
