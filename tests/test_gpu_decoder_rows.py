"""esb_rmsnorm and esb_swiglu against their definitions in 64 bits.

Tolerances (fp32 work, u = 2^-24 per rounding).  Norm: z one rounding, which also enters rstd;
rstd two (its fp64 value rounded once, one spare); two products: 6 u.  Gated activation: the
exponential within 4 u, 1 + e one, the quotient 3, its product one, the last one: 12 u, and an
absolute floor where 1 + e passes the range of a reciprocal (|gate| > 87: the value is below 2^-119
of up).  Outputs add one rounding to their type (tests/decoder_ref.py)."""
import pytest
import torch

import decoder_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NORM_REL, GATE_REL, GATE_FLOOR = 6 * U, 12 * U, 2.0 ** -119
EPS = 1e-5


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def make(seed, rows, d, dtype, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, d, generator=g) * torch.exp(spread * torch.randn(d, generator=g))
    return x.to(dtype)


SIZES = [(1, 1), (3, 7), (2, 8), (5, 63), (4, 64), (3, 65), (7, 511), (2, 512), (3, 513), (9, 1000),
         (2, 1024), (2, 1031), (1, 2048), (3, 2049), (1, 4096), (2, 4100), (2, 8192), (2, 9216),
         (1, 16384), (2, 16391), (1, 32768), (1, 40001), (1, 65536), (300, 129)]


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_norm(esb, rows, d, t):
    dtype = ref.TYPES[t]
    log("norm rows=%d d=%d %s" % (rows, d, t))
    x, r = make(d, rows, d, dtype, 0.3), make(d + 1, rows, d, dtype, 0.3)
    w = 1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(3))
    z, y = ref.rmsnorm(x, w, EPS, r)
    gz, gy, g8, gs = esb.esb_rmsnorm(x.cuda(), w.cuda(), EPS, residual=r.cuda(), want_sum=True,
                                     want_y=True)
    ref.check_float(gz, z, U)
    ref.check_float(gy, y, NORM_REL)
    ref.check_e4m3(g8, gs, y, NORM_REL)
    # no residual, no weights, one output at a time: the same bits where the inputs are the same
    z, y = ref.rmsnorm(x, None, EPS)
    none, gy, n8, ns = esb.esb_rmsnorm(x.cuda(), None, EPS, want_y=True, want_y8=False)
    assert none is None and n8 is None and ns is None
    ref.check_float(gy, y, NORM_REL)
    _, ny, g8, gs = esb.esb_rmsnorm(x.cuda(), None, EPS)
    assert ny is None
    ref.check_e4m3(g8, gs, y, NORM_REL)


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_swiglu(esb, rows, d, t):
    dtype = ref.TYPES[t]
    log("swiglu rows=%d d=%d %s" % (rows, d, t))
    g, u = make(d, rows, d, dtype, 0.5), make(d + 1, rows, d, dtype, 0.3)
    y = ref.swiglu(g, u)
    # the two halves of one buffer, as a gate|up product leaves them
    gu = torch.cat([g, u], 1).cuda()
    gy, g8, gs = esb.esb_swiglu(gu[:, :d], gu[:, d:], want_y=True)
    floor = GATE_FLOOR * float(u.double().abs().max())
    ref.check_float(gy, y, GATE_REL, floor)
    ref.check_e4m3(g8, gs, y, GATE_REL, floor)


def test_swiglu_whole_range(esb):
    g = torch.cat([torch.linspace(-130, 130, 5001), torch.logspace(-38, 2, 500), -torch.logspace(-38, 2, 500)])
    u = torch.full_like(g, 1.0)
    gy, _, _ = esb.esb_swiglu(g[None].cuda(), u[None].cuda(), want_y=True, want_y8=False)
    ref.check_float(gy, ref.swiglu(g[None], u[None]), GATE_REL, GATE_FLOOR)
    inf = float("inf")
    g = torch.tensor([[inf, -inf, float("nan"), 0.0, 3e38, -3e38, 1.0]])
    gy, g8, gs = esb.esb_swiglu(g.cuda(), torch.ones(1, 7).cuda(), want_y=True)
    got = gy.cpu()[0].tolist()
    assert got[0] == inf and got[1] != got[1] and got[2] != got[2] and got[3] == 0
    assert got[4] == pytest.approx(3e38, rel=1e-6) and got[5] == 0
    assert bool(torch.isnan(gs).all()) and bool(torch.isnan(g8.float()).all())


def test_special_rows(esb):
    """Rows of zeros, of the largest values, with NaN and infinities: each row by itself."""
    d = 100
    x = make(5, 8, d, torch.float32)
    x[1] = 0
    x[2] = 3e38          # squares beyond fp32
    x[3, 17] = float("nan")
    x[4, 99] = float("inf")
    x[5] = 1e-38
    x[6] = 0
    x[6, 3] = -1e-30
    _, gy, g8, gs = esb.esb_rmsnorm(x.cuda(), None, EPS, want_y=True)
    for i in (0, 1, 2, 5, 6, 7):
        _, y = ref.rmsnorm(x[i:i + 1], None, EPS)
        # rstd of row 2 is a subnormal number of 2^-128: 21 bits
        rel = 2.0 ** -20 if i == 2 else NORM_REL
        ref.check_float(gy[i:i + 1], y, rel, 2.0 ** -149)
        ref.check_e4m3(g8[i:i + 1], gs[i:i + 1], y, rel, 2.0 ** -149)
    assert float(gs[1]) == 2.0 ** -126 and not bool(g8[1].float().any())
    for i in (3, 4):
        assert bool(torch.isnan(gs[i])) and bool(torch.isnan(g8[i].float()).all())
    assert bool(torch.isnan(gy[3]).all())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,shift", [(1000, 0), (1000, 3), (1031, 1), (4096, 5)])
def test_pitches_and_alignment(esb, t, d, shift):
    """Rows apart, starting at any element; nothing outside the rows is written."""
    dtype, rows = ref.TYPES[t], 5
    ld = d + 13
    base = [make(20 + i, rows, ld, dtype, 0.2) for i in range(2)]
    flat = [torch.cat([torch.full((shift,), float("nan")).to(dtype), b.reshape(-1)]).cuda() for b in base]
    x, r = [f[shift:].view(rows, ld)[:, :d] for f in flat]
    out = [torch.full((rows * ld + shift,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    s_out, y_out = [o[shift:].view(rows, ld)[:, :d] for o in out]
    b8 = torch.full((rows * ld + shift,), 7.0, dtype=torch.float32, device="cuda").to(torch.float8_e4m3fn)
    y8 = b8[shift:].view(rows, ld)[:, :d]
    w = 1 + 0.1 * torch.randn(d + 1, generator=torch.Generator().manual_seed(1))
    wd = w.cuda()[1:]
    z, y = ref.rmsnorm(base[0][:, :d], w[1:], EPS, base[1][:, :d])
    got = esb.esb_rmsnorm(x, wd, EPS, residual=r, sum_out=s_out, y=y_out, y8=y8)
    assert got[0] is s_out and got[1] is y_out and got[2] is y8
    ref.check_float(s_out, z, U)
    ref.check_float(y_out, y, NORM_REL)
    ref.check_e4m3(y8, got[3], y, NORM_REL)
    for o in out + [b8]:
        o = o.float()
        assert bool((o[:shift] == 7).all())
        assert bool((o[shift:].view(rows, ld)[:, d:] == 7).all())


def test_in_place(esb):
    x, r = make(1, 33, 700, torch.bfloat16), make(2, 33, 700, torch.bfloat16)
    xd, rd = x.cuda(), r.cuda()
    a = esb.esb_rmsnorm(xd, None, EPS, residual=rd, want_sum=True, want_y=True)
    s, y, y8, sc = esb.esb_rmsnorm(xd, None, EPS, residual=rd, sum_out=rd, y=xd)
    assert s is rd and y is xd
    for p, q in zip(a, (s, y, y8, sc)):
        assert torch.equal(p.float(), q.float())
    g, u = make(3, 9, 300, torch.float16), make(4, 9, 300, torch.float16)
    gd, ud = g.cuda(), u.cuda()
    want = esb.esb_swiglu(gd, ud, want_y=True, want_y8=False)[0]
    assert torch.equal(esb.esb_swiglu(gd, ud, y=gd, want_y8=False)[0], want)


def test_offsets_beyond_32_bits(esb):
    """Rows whose byte and element offsets pass 2^32 (bf16, pitch 2^27)."""
    rows, d, ld = 34, 200, 1 << 27
    buf = torch.empty(((rows - 1) * ld + d,), dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, d), (ld, 1))
    h = make(9, rows, d, torch.bfloat16)
    x.copy_(h)
    _, y = ref.rmsnorm(h, None, EPS)
    _, gy, g8, gs = esb.esb_rmsnorm(x, None, EPS, want_y=True)
    ref.check_float(gy, y, NORM_REL)
    ref.check_e4m3(g8, gs, y, NORM_REL)
    esb.esb_rmsnorm(x, None, EPS, y=x, want_y8=False)
    assert torch.equal(x.cpu(), gy.cpu())


def test_many_rows(esb):
    """More rows than one launch's workgroups."""
    rows, d = (1 << 21) + 3, 2
    x = make(4, rows, d, torch.bfloat16)
    _, gy, _, gs = esb.esb_rmsnorm(x.cuda(), None, EPS, want_y=True)
    _, y = ref.rmsnorm(x, None, EPS)
    ref.check_float(gy, y, NORM_REL)


def test_nothing_to_do(esb):
    for rows, d in ((0, 64), (3, 0)):
        x = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
        _, y, y8, s = esb.esb_rmsnorm(x, None, EPS, want_y=True)
        assert y.shape == y8.shape == (rows, d) and s.shape == (rows,)
        assert esb.esb_swiglu(x, x, want_y=True)[0].shape == (rows, d)


def test_streams(esb):
    """Work on a stream other than the current one, ordered after what that stream holds."""
    x = make(6, 50, 640, torch.bfloat16)
    xd = torch.zeros(50, 640, dtype=torch.bfloat16, device="cuda")
    want = esb.esb_rmsnorm(x.cuda(), None, EPS, want_y=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        xd.copy_(x.cuda())
    got = esb.esb_rmsnorm(xd, None, EPS, want_y=True, stream=s)
    s.synchronize()
    for p, q in zip(want[1:], got[1:]):
        assert torch.equal(p.float(), q.float())


def test_refusals(esb):
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(esb.EsbError):
        esb.esb_rmsnorm(x, None, 0.0)
    with pytest.raises(esb.EsbError):
        esb.esb_rmsnorm(x, None, EPS, want_y8=False)            # no output
    with pytest.raises(esb.EsbError):
        esb.esb_rmsnorm(torch.zeros(1, 65537, device="cuda"), None, EPS)
    with pytest.raises(TypeError):
        esb.esb_rmsnorm(x.cpu(), None, EPS)
    with pytest.raises(TypeError):
        esb.esb_rmsnorm(x.double(), None, EPS)
    with pytest.raises(ValueError):
        esb.esb_rmsnorm(x.t(), None, EPS)
    with pytest.raises(ValueError):
        esb.esb_rmsnorm(x, torch.ones(63, device="cuda"), EPS)
    with pytest.raises(ValueError):
        esb.esb_rmsnorm(x, None, EPS, residual=x[:, :32])
    with pytest.raises(ValueError):
        esb.esb_rmsnorm(x, None, EPS, residual=x.float())
    with pytest.raises(ValueError):
        esb.esb_rmsnorm(x[:1].expand(4, 64), None, EPS)
    with pytest.raises(ValueError):
        esb.esb_swiglu(x, x[:3])


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_strongly_negative_gates(esb, t):
    """Gates far below zero: small values, but whole ones, and a large `up` makes them large again.
    The tolerance has no floor but half the output type's smallest step."""
    dtype = ref.TYPES[t]
    top = 6e4 if t == "f16" else 3e38
    ups = [1.0, -1.0, 1e-4, 1e4, top] + ([2.0 ** 100, 1e-20, 1e-38] if t != "f16" else [])
    g = torch.linspace(-260, -55, 821).to(dtype)
    rows = [(g[i:i + 411], torch.full((411,), u).to(dtype)) for u in ups for i in (0, 410)]
    g, u = [torch.stack(v) for v in zip(*rows)]
    # one such gate among ordinary ones
    g = torch.cat([g, torch.linspace(-4, 4, 411).to(dtype)[None]])
    g[-1, 200] = -88.0
    u = torch.cat([u, torch.full((1, 411), top / 8).to(dtype)])
    y = ref.swiglu(g, u)
    gy, g8, gs = esb.esb_swiglu(g.cuda(), u.cuda(), want_y=True)
    ref.check_float(gy, y, GATE_REL)
    assert float((gy[:, 0] != 0).sum()) >= 2 or t == "f16"
    # bytes: where the row's largest value is a normal number
    big = y.abs().amax(1) > 2.0 ** -110
    ref.check_e4m3(g8[big.cuda()], gs[big.cuda()], y[big], GATE_REL, 2.0 ** -149)


def test_stream_arguments(esb):
    """What names a stream in this binding: a torch stream, its handle (0: the default stream) and any
    object that holds one."""
    x = make(8, 20, 384, torch.bfloat16).cuda()
    want = esb.esb_rmsnorm(x, None, EPS)
    w4 = esb.esb_w4_quantize(x, 32)
    gate, (q, alpha) = esb.esb_swiglu(x, x), esb.esb_w4_unpack(w4, 20, 384, 32)
    y = esb.esb_w4_gemm(x, w4, 20, 32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    class Holder:
        cuda_stream = side.cuda_stream

    for stream in (side, side.cuda_stream, Holder(), 0, torch.cuda.default_stream()):
        got = esb.esb_rmsnorm(x, None, EPS, stream=stream)
        g = esb.esb_swiglu(x, x, stream=stream)
        v4 = esb.esb_w4_quantize(x, 32, stream=stream)
        v, a = esb.esb_w4_unpack(w4, 20, 384, 32, stream=stream)
        p = esb.esb_w4_gemm(x, w4, 20, 32, stream=stream)
        torch.cuda.synchronize()
        for s, t in zip(want[2:] + gate[1:] + (w4, q, alpha, y), got[2:] + g[1:] + (v4, v, a, p)):
            assert torch.equal(s.view(torch.uint8) if s.dtype.itemsize == 1 else s,
                               t.view(torch.uint8) if t.dtype.itemsize == 1 else t)
