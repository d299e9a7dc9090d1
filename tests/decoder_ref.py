"""Definitions of the decoder operators in 64 bits (torch on the CPU), for their GPU tests."""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# unit roundoff of one rounding to the type, and half its smallest step
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
LEVELS = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
# ESB(4,1) code -> value: sign | two exponent bits (all ones: subnormal) | one fraction bit
CODE_VALUES = torch.tensor([1, 1.5, 2, 3, 4, 6, 0, .5, -1, -1.5, -2, -3, -4, -6, -0., -.5],
                           dtype=torch.float64)


def rmsnorm(x, w, eps, residual=None):
    z = x.double()
    if residual is not None:
        z = z + residual.double()
    y = z / torch.sqrt(z.square().mean(1, keepdim=True) + eps)
    return z, y if w is None else y * w.double()


def swiglu(gate, up):
    g = gate.double()
    return g / (1 + torch.exp(-g)) * up.double()


def row_scale(y):
    return (y.abs().amax(1) / 448).clamp(min=2.0 ** -126)


def check_float(got, ref, rel, floor=0.0):
    """got (any float type) against the exact ref: rel * |ref| + floor of fp32 work, then one
    rounding to got's type."""
    u, step = ROUND[got.dtype], STEP[got.dtype]
    off = (got.double().cpu() - ref).abs()
    allowed = (rel + u * (1 + rel)) * ref.abs() + step + floor
    assert bool((off <= allowed).all()), (off / allowed.clamp(min=1e-300)).max()


def check_e4m3(byte, scale, ref, rel, floor=0.0):
    """8-bit rows: the scale of the exact row, and the nearest E4M3 value of ref / scale, with the
    fp32 error `rel` (and `floor`, absolute) of the value that was rounded."""
    s = scale.double().cpu()
    want = row_scale(ref)
    assert bool(((s - want).abs() <= (rel + 2.0 ** -23) * want + floor / 448 + 2.0 ** -149).all())
    v = ref / s[:, None]
    e = torch.frexp(v)[1] - 1
    half = torch.ldexp(torch.ones_like(v), e.clamp(min=-6) - 4)
    off = (byte.cpu().double() - v).abs()
    allowed = half + (rel + 2.0 ** -22) * v.abs() + floor / s[:, None]
    assert bool((off <= allowed).all()), (off / allowed).max()


def quantize(w, group, factors):
    """(values, scales): w N x K; the candidate of the least squared error per group."""
    N, K = w.shape
    groups = -(-K // group)
    q = torch.zeros(N, K, dtype=torch.float64)
    alpha = torch.zeros(N, groups, dtype=torch.float64)
    mids = (LEVELS[1:] + LEVELS[:-1]) / 2
    for g in range(groups):
        b = w[:, g * group:(g + 1) * group]
        top = b.abs().float().amax(1)
        least = torch.full((N,), float("inf"), dtype=torch.float64)
        b = b.double()
        for f in factors:
            f32 = torch.tensor(f, dtype=torch.float32)
            if not (f32 > 0 and torch.isfinite(f32)):
                continue
            a = (top * f32 / 6).clamp(min=2.0 ** -126).to(torch.bfloat16).double()
            v = LEVELS[torch.bucketize(b.abs() / a[:, None], mids, right=True)]
            v = torch.where(b < 0, -v, v)
            err = (b - a[:, None] * v).square().sum(1)
            take = (err < least) & torch.isfinite(a)
            least = torch.where(take, err, least)
            alpha[:, g] = torch.where(take, a, alpha[:, g])
            q[:, g * group:(g + 1) * group] = torch.where(take[:, None], v, q[:, g * group:(g + 1) * group])
    return q, alpha


def dequantize(q, alpha, group):
    return q * alpha.repeat_interleave(group, 1)[:, :q.shape[1]]
