"""esb_w4_gemm on 8-bit rows whose products span the whole range of E4M3 times E2M1 (2^-10 to 2688).

Every product counts, whatever stands beside it: the tolerance is that of fp32 sums alone,
(K + groups + 4) 2^-24 S with S = s_m sum_k |x| alpha |q| of that output, then one rounding to the
output's type.  It holds for a row alone and among others, for every group and output type."""
import pytest
import torch

import decoder_ref as ref
from gpuutil import log, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn


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


def check(y, x, s, codes, alpha, group):
    K = x.shape[1]
    w = ref.dequantize(ref.CODE_VALUES[codes.long()], alpha.double(), group)
    xd = x.double() * s.double()[:, None]
    want = xd @ w.t()
    allowed = (K + alpha.shape[1] + 4) * U * (xd.abs() @ w.abs().t())
    allowed = allowed * (1 + ref.ROUND[y.dtype]) + ref.ROUND[y.dtype] * want.abs() + ref.STEP[y.dtype]
    off = (y.double().cpu() - want).abs()
    assert bool((off <= allowed).all()), (off / allowed).max()


def massive(M, K, seed):
    """A few channels hundreds of times the others, as a norm hands them over."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(M, K, generator=g)
    v[:, torch.randperm(K, generator=g)[:max(1, K // 256)]] *= 400
    s = v.abs().amax(1) / 448
    return (v / s[:, None]).to(E4M3), s


@pytest.mark.parametrize("M", [1, 3, 20, 64, 150, 600])
@pytest.mark.parametrize("N,K", [(200, 640), (1030, 2304), (100, 333)])
@pytest.mark.parametrize("y", ["bf16", "f16", "f32"])
def test_massive_channels(esb, M, N, K, y):
    log("w4 gemm outliers M=%d N=%d K=%d %s" % (M, N, K, y))
    x, s = massive(M, K, M + K)
    for group in (32, 64, 128):
        codes, alpha = weights(N + group, N, K, group)
        w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
        check(esb.esb_w4_gemm(x.cuda(), w4, N, group, x_scale=s.cuda(), y_dtype=ref.TYPES[y]), x, s,
              codes, alpha, group)


@pytest.mark.parametrize("M", [1, 3, 20, 64, 150, 600])
@pytest.mark.parametrize("y", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pad", [0, 5])
def test_outliers_that_cancel(esb, M, y, pad):
    """448 and -448 under equal weights beside values of at most 2^-4: the output is theirs alone."""
    N, K = 150, 256 + pad
    log("w4 gemm cancelling outliers M=%d K=%d %s" % (M, K, y))
    g = torch.Generator().manual_seed(M)
    v = (torch.rand(M, K, generator=g) - 0.5) / 8
    for m in range(M):
        for k in range(0, 256, 64):                 # in every 64 columns
            i, j = (k + torch.randperm(64, generator=g)[:2]).tolist()
            v[m, i], v[m, j] = 448, -448
    x, s = v.to(E4M3), torch.rand(M, generator=g) + 0.5
    for group in (32, 64, 128):
        codes, alpha = weights(group, N, K, group)
        codes[:, :256] = codes[:, :256:64].repeat_interleave(64, 1)
        w4 = esb.esb_w4_pack(codes.cuda(), alpha.cuda(), group)
        check(esb.esb_w4_gemm(x.cuda(), w4, N, group, x_scale=s.cuda(), y_dtype=ref.TYPES[y]), x, s,
              codes, alpha, group)
