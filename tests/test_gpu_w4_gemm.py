"""esb_w4_gemm against the definition in 64 bits.

Tolerance per output, from S = s_m sum_k |x| alpha |q| of that output: fp32 sums of K products and
ceil(K / group) scaled partial sums, each addition within 2^-24 of the running sum, which S bounds:
(K + groups + 4) 2^-24 S, then one rounding to the output's type.  With 8-bit activations and a
16-bit output a matrix instruction may drop products below 2^-13 of its largest, of 128: at most
128 2^-13 of the largest |x| alpha |q| in every 128 columns is added for those."""
import pytest
import torch

import decoder_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
XT = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": E4M3}


@pytest.fixture(scope="module")
def esb():
    torch_cuda()
    from paper_2109_03513_amd import esb as e
    e.lib()
    return e


def weights(seed, N, K, group):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 16, (N, K), generator=g, dtype=torch.uint8)
    alpha = (0.01 * torch.exp(torch.randn(N, -(-K // group), generator=g))).to(torch.bfloat16)
    return codes, alpha


def acts(seed, M, K, x):
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(M, K, generator=g) * torch.exp(0.5 * torch.randn(K, generator=g))
    if x != "e4m3":
        return v.to(XT[x]), None
    s = (v.abs().amax(1) / 448).clamp(min=2.0 ** -126) if K else torch.ones(M)
    return (v / s[:, None]).to(E4M3), s


def check(y, x, s, codes, alpha, group):
    K = x.shape[1]
    w = ref.dequantize(ref.CODE_VALUES[(codes & 15).long()], alpha.double(), group)
    xd = x.double() if s is None else x.double() * s.double()[:, None]
    want = xd @ w.t()
    size = xd.abs() @ w.abs().t()
    allowed = (K + alpha.shape[1] + 4) * U * size
    if x.dtype == E4M3 and y.dtype != torch.float32:
        for k in range(0, K, 128):
            top = xd[:, k:k + 128].abs().amax(1)[:, None] * w[:, k:k + 128].abs().amax(1)[None]
            allowed = allowed + 128 * 2.0 ** -13 * top
    got = y.double().cpu()
    off = (got - want).abs()
    allowed = allowed * (1 + ref.ROUND[y.dtype]) + ref.ROUND[y.dtype] * want.abs() + ref.STEP[y.dtype]
    assert bool((off <= allowed).all()), (off / allowed).max()
    # and on the whole: one rounding to the type, and a part in 2000 for the dropped products
    extra = 5e-4 if x.dtype == E4M3 and y.dtype != torch.float32 else 2e-6
    assert float((got - want).norm()) <= (ref.ROUND[y.dtype] + extra) * float(want.norm()) + 1e-30


SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 129), (3, 100, 31), (1, 257, 1000), (5, 64, 32), (15, 40, 385),
          (16, 33, 640), (17, 48, 256), (31, 130, 777), (33, 512, 128), (48, 96, 2048), (64, 100, 511),
          (65, 65, 65), (100, 300, 1152), (128, 256, 512), (129, 257, 130), (250, 520, 1030),
          (300, 1000, 260), (513, 130, 384), (1, 4096, 2304), (70, 2100, 129), (1025, 320, 192)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"),
                                 ("e4m3", "bf16"), ("e4m3", "f16"), ("e4m3", "f32")])
def test_product(esb, M, N, K, x, y):
    log("w4 gemm M=%d N=%d K=%d %s -> %s" % (M, N, K, x, y))
    xv, s = acts(M + K, M, K, x)
    xd, sd = xv.cuda(), None if s is None else s.cuda()
    for group in (32, 64, 128):
        codes, alpha = weights(N + group, N, K, group)
        w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
        got = esb.esb_w4_gemm(xd, w4, N, group, x_scale=sd, y_dtype=ref.TYPES[y])
        check(got, xv, s, codes, alpha, group)
        assert torch.equal(got, esb.esb_w4_gemm(xd, w4, N, group, x_scale=sd, y_dtype=ref.TYPES[y]))


@pytest.mark.parametrize("M,N,K", [(1, 1500, 4096), (8, 512, 9216), (40, 1024, 2048), (200, 2048, 1024),
                                   (700, 1536, 1100), (2049, 1030, 520)])
@pytest.mark.parametrize("x", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("group", [32, 128])
def test_larger_products(esb, M, N, K, x, group):
    log("w4 gemm M=%d N=%d K=%d %s group=%d" % (M, N, K, x, group))
    xv, s = acts(M + K, M, K, x)
    codes, alpha = weights(N, N, K, group)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
    sd = None if s is None else s.cuda()
    for y in (torch.float32, torch.bfloat16):
        check(esb.esb_w4_gemm(xv.cuda(), w4, N, group, x_scale=sd, y_dtype=y), xv, s, codes, alpha, group)


@pytest.mark.parametrize("M,N,K", [(30, 2000, 9232), (64, 512, 9216), (60, 9190, 4112), (500, 4090, 2064), (520, 4100, 528),
                                   (1000, 4090, 4112), (2000, 4090, 1040), (2040, 4580, 528), (4090, 4090, 528)])
@pytest.mark.parametrize("x", ["bf16", "e4m3"])
@pytest.mark.parametrize("pad,group", [(0, 128), (0, 32), (1, 64)])
def test_tiles(esb, M, N, K, x, pad, group):
    """Sizes that between them take every tile and number of column ranges, rows aligned and not."""
    log("w4 gemm M=%d N=%d K=%d %s pad=%d group=%d" % (M, N, K, x, pad, group))
    xv, s = acts(M + K, M, K, x)
    xd = torch.empty(M, K + pad, dtype=XT[x], device="cuda")[:, :K]
    xd.copy_(xv.cuda())
    codes, alpha = weights(N, N, K, group)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
    check(esb.esb_w4_gemm(xd, w4, N, group, x_scale=None if s is None else s.cuda()), xv, s, codes, alpha, group)


def test_every_row_alike(esb):
    """A row's output does not depend on the other rows of its call, beyond the order of sums."""
    codes, alpha = weights(1, 200, 700, 64)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 64)
    xv, _ = acts(2, 300, 700, "bf16")
    xd = xv.cuda()
    xd[7] = float("nan")
    xd[200, 3] = float("inf")
    y = esb.esb_w4_gemm(xd, w4, 200, 64, y_dtype=torch.float32)
    keep = torch.ones(300, dtype=torch.bool)
    keep[7] = keep[200] = False
    check(y[keep.cuda()], xv[keep], None, codes, alpha, 64)
    assert bool(torch.isnan(y[7]).all()) and not bool(torch.isfinite(y[200]).any())


@pytest.mark.parametrize("M", [3, 40, 300])
def test_rows_without_a_scale(esb, M):
    """8-bit rows of NaN under a NaN scale, as the row operators leave them, and a NaN byte alone."""
    codes, alpha = weights(1, 200, 700, 64)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 64)
    xv, s = acts(2, M, 700, "e4m3")
    xd, sd = xv.cuda(), s.cuda()
    sd[0] = float("nan")
    xd[0].view(torch.uint8).fill_(0x7F)
    xd[2].view(torch.uint8)[699] = 0x7F
    for y in (torch.bfloat16, torch.float32):
        out = esb.esb_w4_gemm(xd, w4, 200, 64, x_scale=sd, y_dtype=y)
        assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[2]).all())
        keep = [i for i in range(M) if i not in (0, 2)]
        check(out[keep], xv[keep], s[keep], codes, alpha, 64)


@pytest.mark.parametrize("K", [2048, 9216])
def test_a_stream_of_its_own(esb, K):
    """Calls on another stream than the current one: outputs and workspace belong to it."""
    codes, alpha = weights(1, 512, K, 128)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 128)
    xv, _ = acts(3, 64, K, "bf16")
    x = xv.cuda()
    assert K < 9216 or esb.esb_w4_gemm_workspace_size(64, 512, K, 128, 1, 1) > 0
    want = esb.esb_w4_gemm(x, w4, 512, 128)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for _ in range(20):
            got = esb.esb_w4_gemm(x, w4, 512, 128, stream=stream)
            junk = torch.full((1 << 20,), float("nan"), device="cuda")       # the current stream's memory
        side.synchronize()
        assert torch.equal(got, want)
    del junk


@pytest.mark.parametrize("M", [1, 20, 150, 600])
@pytest.mark.parametrize("x", ["bf16", "e4m3"])
def test_groups_without_a_scale_reach_their_outputs_only(esb, M, x):
    codes, alpha = weights(4, 70, 300, 128)
    alpha[5, 1] = float("nan")
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 128)
    xv, s = acts(5, M, 300, x)
    y = esb.esb_w4_gemm(xv.cuda(), w4, 70, 128, x_scale=None if s is None else s.cuda())
    assert bool(torch.isnan(y[:, 5]).all())
    keep = [n for n in range(70) if n != 5]
    check(y[:, keep], xv, s, codes[keep], alpha[keep], 128)


@pytest.mark.parametrize("M", [1, 4, 60, 140, 520])
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_pitches_and_alignment(esb, M, x, y, shift):
    """Rows apart, at any element's alignment, NaN around them; outputs apart, nothing else written."""
    N, K, group = 77, 333, 64
    xv, s = acts(M, M, K, x)
    ldx = K + 11
    buf = torch.full((M * ldx + shift,), float("nan")).to(XT[x])
    view = buf[shift:].view(M, ldx)[:, :K]
    view.copy_(xv)
    codes, alpha = weights(3, N, K, group)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
    xd = buf.cuda()[shift:].view(M, ldx)[:, :K]
    ldy = N + 5
    out = torch.full((M * ldy + shift,), 7.0, dtype=ref.TYPES[y], device="cuda")
    yv = out[shift:].view(M, ldy)[:, :N]
    got = esb.esb_w4_gemm(xd, w4, N, group, x_scale=None if s is None else s.cuda(), y=yv)
    assert got is yv
    check(yv, xv, s, codes, alpha, group)
    assert bool((out[:shift] == 7).all()) and bool((out[shift:].view(M, ldy)[:, N:] == 7).all())


def test_offsets_beyond_32_bits(esb):
    """Activations and outputs whose offsets pass 2^32 elements."""
    N, K, M = 40, 160, 36
    ld = 1 << 27
    codes, alpha = weights(3, N, K, 32)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 32)
    xv, s = acts(1, M, K, "e4m3")
    buf = torch.empty((M - 1) * ld + K, dtype=torch.uint8, device="cuda").view(E4M3)
    xd = buf.as_strided((M, K), (ld, 1))
    xd.copy_(xv.cuda())
    yd = torch.empty((M - 1) * ld + N, dtype=torch.bfloat16, device="cuda").as_strided((M, N), (ld, 1))
    esb.esb_w4_gemm(xd, w4, N, 32, x_scale=s.cuda(), y=yd)
    check(yd, xv, s, codes, alpha, 32)


@pytest.mark.parametrize("M", [1, 20, 150])
@pytest.mark.parametrize("x", ["bf16", "e4m3"])
@pytest.mark.parametrize("K,group", [((1 << 23) + 64, 64), ((1 << 24) + 96, 128)])
def test_long_rows(esb, M, x, K, group):
    """Rows of millions of columns, zeros but for the last ones: those meet their own weights."""
    log("w4 gemm M=%d K=%d %s" % (M, K, x))
    N, at = 40, K // group * group - 2 * group
    g = torch.Generator(device="cuda").manual_seed(M)
    codes = torch.randint(0, 16, (N, K), generator=g, dtype=torch.uint8, device="cuda")
    alpha = (0.01 * (1 + torch.rand(N, -(-K // group), generator=g, device="cuda"))).to(torch.bfloat16)
    w4 = esb.esb_w4_pack(codes, alpha, group)
    xv, s = acts(M, M, K - at, x)
    xd = torch.zeros(M, K, dtype=torch.uint8 if x == "e4m3" else XT[x], device="cuda").view(XT[x])
    xd[:, at:] = xv.cuda()
    y = esb.esb_w4_gemm(xd, w4, N, group, x_scale=None if s is None else s.cuda())
    check(y, xv, s, codes[:, at:].cpu(), alpha[:, at // group:].cpu(), group)


def test_weights_beyond_32_bits(esb):
    """Packed weights of more than 2^32 bytes: the last rows read their own tiles."""
    N, K, group = 270016, 32768, 128
    w4 = torch.zeros(esb.esb_w4_size(N, K, group), dtype=torch.uint8, device="cuda")
    assert w4.numel() > 1 << 32
    codes, alpha = weights(8, 32, K, group)
    part = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
    tiles, chunks, groups = 1, K // 64, K // 128
    first = (N // 32 - tiles) * chunks
    w4[1024 * first:1024 * (first + tiles * chunks)] = part[:1024 * tiles * chunks]
    w4[w4.numel() - 64 * tiles * groups:] = part[1024 * tiles * chunks:]
    for M, x in ((1, "bf16"), (40, "e4m3"), (300, "bf16"), (300, "e4m3")):
        xv, s = acts(2, M, K, x)
        y = esb.esb_w4_gemm(xv.cuda(), w4, N, group, x_scale=None if s is None else s.cuda())
        assert not bool(y[:, :N - 32].any())
        check(y[:, N - 32:], xv, s, codes, alpha, group)


@pytest.mark.parametrize("M,N,K,x,group", [(20, 300, 520, "bf16", 64), (64, 512, 2048, "f16", 32),
                                           (64, 512, 9216, "f16", 32), (30, 300, 9216, "e4m3", 128),
                                           (130, 257, 333, "bf16", 128), (150, 300, 777, "e4m3", 128),
                                           (140, 200, 640, "e4m3", 32)])
def test_with_and_without_workspace(esb, M, N, K, x, group):
    """The C entry without a workspace, and with one full of NaN: both right, nothing written past it."""
    L = esb.lib()
    xv, s = acts(M, M, K, x)
    xd, sd = xv.cuda(), None if s is None else s.cuda()
    codes, alpha = weights(N, N, K, group)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
    tx = {"bf16": 1, "f16": 2, "e4m3": 3}[x]
    need = L.esb_w4_gemm_workspace_size(M, N, K, group, tx, 1)
    for ws in (None, torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")):
        if ws is not None and need == 0:
            continue
        y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        st = L.esb_w4_gemm(M, N, K, group, xd.data_ptr(), K, tx, None if sd is None else sd.data_ptr(),
                           w4.data_ptr(), y.data_ptr(), N, 1, None if ws is None else ws.data_ptr(), need,
                           torch.cuda.current_stream().cuda_stream)
        assert st == 0
        check(y, xv, s, codes, alpha, group)
        assert ws is None or bool((ws[need:] == 0xFF).all())


def test_empty(esb):
    codes, alpha = weights(1, 20, 64, 32)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 32)
    assert esb.esb_w4_gemm(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), w4, 20, 32).shape == (0, 20)
    none = torch.empty(1, dtype=torch.uint8, device="cuda")
    y = torch.full((3, 20), 5.0, dtype=torch.bfloat16, device="cuda")
    esb.esb_w4_gemm(torch.empty(3, 0, dtype=torch.bfloat16, device="cuda"), none, 20, 32, y=y)
    assert not bool(y.any())


def test_streams_and_graph(esb):
    """On a stream of its own, and captured and replayed with new activations."""
    codes, alpha = weights(1, 300, 512, 128)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 128)
    for M in (1, 40, 300):
        xs = [acts(i, M, 512, "bf16")[0].cuda() for i in range(3)]
        want = [esb.esb_w4_gemm(x, w4, 300, 128) for x in xs]
        x, y = torch.zeros_like(xs[0]), torch.zeros_like(want[0])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            x.copy_(xs[0])
            esb.esb_w4_gemm(x, w4, 300, 128, y=y)
        side.synchronize()
        assert torch.equal(y, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            esb.esb_w4_gemm(x, w4, 300, 128, y=y)
        for v, e in zip(xs, want):
            x.copy_(v)
            graph.replay()
            assert torch.equal(y, e)
            torch.cuda.synchronize()
            assert torch.equal(esb.esb_w4_gemm(v, w4, 300, 128), e)


def test_refusals(esb):
    codes, alpha = weights(1, 20, 64, 32)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 32)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(esb.EsbError):
        esb.esb_w4_gemm(x.float(), w4, 20, 32)                       # fp32 activations
    with pytest.raises(esb.EsbError):
        esb.esb_w4_gemm(x, w4, 20, 48)
    with pytest.raises(esb.EsbError):
        esb.esb_w4_gemm(x, w4, 2000, 32)                             # weights of another matrix
    with pytest.raises(TypeError):
        esb.esb_w4_gemm(x.cpu(), w4, 20, 32)
    with pytest.raises(ValueError):
        esb.esb_w4_gemm(x.t(), w4, 20, 32)
    with pytest.raises(ValueError):
        esb.esb_w4_gemm(x, w4, 20, 32, x_scale=torch.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        esb.esb_w4_gemm(x, w4, 20, 32, y=torch.zeros(2, 21, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        esb.esb_w4_gemm(x, w4, 20, 32, y_dtype=torch.int32)


@pytest.mark.parametrize("M", [1, 3, 17, 40, 128, 300])
@pytest.mark.parametrize("x", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("y", ["bf16", "f16", "f32"])
def test_no_columns(esb, M, x, y):
    """K = 0 writes zeros, and them only, whatever the rows' scales hold."""
    N = 77
    none = torch.empty(1, dtype=torch.uint8, device="cuda")
    xd = torch.empty(M, 0, dtype=XT[x], device="cuda")
    s = torch.full((M,), float("nan"), device="cuda")
    for group in (32, 64, 128):
        for scale in (None, s):
            out = torch.full((M, N + 5), 7.0, dtype=ref.TYPES[y], device="cuda")
            esb.esb_w4_gemm(xd, none, N, group, x_scale=scale, y=out[:, :N])
            assert not bool(out[:, :N].any()) and bool((out[:, N:] == 7).all())


def test_workspaces_that_the_kernels_cannot_write(esb):
    codes, alpha = weights(1, 512, 9216, 128)
    w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), 128)
    x = acts(2, 64, 9216, "bf16")[0].cuda()
    need = esb.esb_w4_gemm_workspace_size(64, 512, 9216, 128, 1, 1)
    with pytest.raises(TypeError):
        esb.esb_w4_gemm(x, w4, 512, 128, workspace=torch.empty(need, dtype=torch.uint8))
    with pytest.raises(TypeError):
        esb.esb_w4_gemm(x, w4, 512, 128, workspace=torch.empty(need, dtype=torch.uint8).numpy())
    room = torch.zeros(2 * need, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        esb.esb_w4_gemm(x, w4, 512, 128, workspace=room[::2])
    with pytest.raises(esb.EsbError):
        esb.esb_w4_gemm(x, w4, 512, 128, workspace=room[:need - 1])
    assert not bool(room.any())
    want = esb.esb_w4_gemm(x, w4, 512, 128)
    assert torch.equal(esb.esb_w4_gemm(x, w4, 512, 128, workspace=room[:need]), want)


@pytest.mark.parametrize("M", [1, 7, 20, 64, 150, 600])
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("K", [300, 704, 9216, 9152])
def test_infinite_scales(esb, M, x, y, K):
    """An infinite scale reaches its outputs only; where it meets a whole group's sum (groups of 32 and
    64), they are infinite with that sum's sign, whatever steps a tile or a range of columns adds."""
    log("w4 gemm infinite scale M=%d K=%d %s" % (M, K, x))
    N = 70
    xv, s = acts(5, M, K, x)
    for group in (32, 64, 128):
        codes, alpha = weights(4, N, K, group)
        groups = alpha.shape[1]
        # the last group, and one within (a sum of +-8 steps at least: no cancellation to zero)
        at = {5: groups - 1, 66: groups // 2, 40: 0}
        for n, g in at.items():
            alpha[n, g] = float("inf")
        w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
        out = esb.esb_w4_gemm(xv.cuda(), w4, N, group, x_scale=None if s is None else s.cuda(),
                              y_dtype=ref.TYPES[y]).cpu()
        q = ref.CODE_VALUES[codes.long()]
        for n, g in at.items():
            c = slice(g * group, min((g + 1) * group, K))
            part = xv[:, c].double() @ q[n, c]
            sure = part.abs() > 1e-3 * (xv[:, c].double().abs() @ q[n, c].abs())
            assert not bool(torch.isfinite(out[:, n]).any())
            if group < 128:
                want = torch.copysign(torch.full((M,), float("inf"), dtype=torch.float64), part)
                assert torch.equal(out[:, n].double()[sure], want[sure]), (n, g)
        keep = [n for n in range(N) if n not in at]
        check(out[:, keep], xv, s, codes[keep], alpha[keep], group)
