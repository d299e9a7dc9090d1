"""esb_kv4_attention where queries, keys and values lie far apart: zeros, the least scales, and scales of
one key, value or group far above another's, seen or not.

Tolerances: those of test_gpu_kv4_attention, which say nothing of a range; what lies behind a query's last
key enters none of them."""
import pytest
import torch

import attention_ref as ref
from gpuutil import log
from test_gpu_kv4_attention import Cache, esb, queries, verify  # noqa: F401

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
