"""esb_attention at the ends of its types.  Tolerances as in test_gpu_attention."""
import pytest
import torch

import attention_ref as ref
from test_gpu_attention import esb, make, starts  # noqa: F401

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def verify(q, k, v, out, causal=True, scale=None):
    """One sequence.  A weight below fp32's smallest normal number, beside a largest one of at least 1, may count
    as zero: that is 2^-126 of the sum of |v|."""
    n, m, d = q.shape[0], k.shape[0], q.shape[2]
    last = torch.arange(n) + m - n if causal else torch.full((n,), m - 1)
    want = ref.attend(q, k, v, last, d ** -0.5 if scale is None else scale)
    ref.check(out, *want, keys=m, d=d, p_round=ref.ROUND[q.dtype],
              p_step=2.0 ** -25 if q.dtype == torch.float16 else 2.0 ** -126)


@pytest.mark.parametrize("power", [10, 18, 24, 32, 60])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n", [150, 1200])
def test_large_scores(esb, power, d, n):  # noqa: F811
    """Scores of about 2^power, finite: the largest takes all, and nothing is NaN."""
    q, k, v = (make(s, n, h, d, dtype=BF16) for s, h in ((46, 2), (47, 1), (48, 1)))
    k = (k.double() * 2.0 ** power).to(BF16)
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n])))
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n]), causal=False), causal=False)


@pytest.mark.parametrize("power", [18, 30])
def test_large_scores_f16(esb, power):  # noqa: F811
    n = 300
    q, k, v = (make(s, n, h, 64, dtype=torch.float16) for s, h in ((46, 2), (47, 1), (48, 1)))
    q, k = ((x.double() * 2.0 ** (power // 2 - 3)).to(torch.float16) for x in (q, k))
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n])))


@pytest.mark.parametrize("power", [100, 118, 122, 126])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n", [150, 1200])
def test_largest_values(esb, power, d, n):  # noqa: F811
    """Values near the end of bf16 under weights that grow by less than 2^8: outputs are finite."""
    up = torch.arange(n, device="cuda").float() / n
    k = up[:, None, None].expand(n, 1, d).to(BF16).contiguous()
    v = torch.where(torch.arange(n, device="cuda") % 200 == 110, 2.0 ** power, 2.0 ** (power - 11))
    v = v[:, None, None].expand(n, 1, d).to(BF16).contiguous()
    q = torch.full((n, 2, d), 5.4 / d, dtype=BF16, device="cuda")
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n]), scale=1.0), scale=1.0)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_smallest_values(esb, d):  # noqa: F811
    n = 300
    q, k, v = (make(s, n, h, d, dtype=BF16) for s, h in ((43, 2), (44, 1), (45, 1)))
    v = (v.double() * 2.0 ** -120).to(BF16)
    verify(q, k, v, esb.esb_attention(q, k, v, starts([n])))


@pytest.mark.parametrize("d", [8, 40, 64, 80, 96, 120, 128, 136, 192, 248, 256])
@pytest.mark.parametrize("pitched", [False, True])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_keys_of_minus_infinity(esb, d, pitched, t):  # noqa: F811
    """A key whose score is -infinity drops out wherever in the head its infinity lies; +infinity is NaN."""
    n, dtype = 150, ref.TYPES[t]
    q, k, v = (make(s, n, h, d, dtype=dtype) for s, h in ((40, 2), (41, 1), (42, 1)))
    q = q.abs() + 0.5
    for at, where, value in ((0, d - 1, -1), (70, d - 8, -1), (100, d - 3, -1), (101, 0, -1), (147, d - 1, 1)):
        k[at, 0, where] = value * float("inf")
    if pitched:      # rows that are not aligned
        wide = torch.zeros(n, d + 1, dtype=dtype, device="cuda")
        wide[:, 1:] = k[:, 0]
        k = wide[:, None, 1:]
    out = esb.esb_attention(q, k, v, starts([n])).cpu()
    want = ref.attend(q.cpu(), k.cpu(), v.cpu(), torch.arange(n), d ** -0.5)[0]
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert bool(torch.isnan(out[0]).all()) and not bool(torch.isnan(out[1:147]).any()) and bool(torch.isnan(out[147:]).all())
    # without those keys the others' weights are the same
    keep = [i for i in range(147) if i not in (0, 70, 100, 101)]
    for i in (120, 146):
        seen = [j for j in keep if j <= i]
        o = ref.attend(q[i:i + 1], k[seen], v[seen], torch.tensor([len(seen) - 1]), d ** -0.5)
        ref.check(out[i:i + 1].cuda(), *o, keys=len(seen), d=d, p_round=ref.ROUND[dtype],
                  p_step=2.0 ** -25 if t == "f16" else 0.0)
