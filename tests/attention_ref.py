"""Definitions of a decoder's attention operators in 64 bits (torch, on the tensors' device)."""
import torch

from decoder_ref import LEVELS, ROUND, STEP, TYPES  # noqa: F401

U = 2.0 ** -24                       # one rounding to fp32


def table(rows, rot, base=10000.0):
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    a = torch.arange(rows, dtype=torch.float64)[:, None] * f
    return torch.cat([torch.cos(a), torch.sin(a)], 1).float()


def turn(x, w, eps, tab, positions, adjacent):
    """(y, size): heads [tokens, heads, d] normed and rotated, and the magnitudes |a c| + |b s| that
    the errors of fp32 work are relative to."""
    y = x.double()
    if eps > 0:
        y = y / torch.sqrt(y.square().mean(2, keepdim=True) + eps)
        if w is not None:
            y = y * w.double()
    if tab is None or tab.shape[1] == 0:
        return y, y.abs()
    rot = tab.shape[1]
    h = rot // 2
    row = tab.double()[positions.long()][:, None]
    c, s = row[..., :h], row[..., h:]
    i = torch.arange(h)
    ia, ib = (2 * i, 2 * i + 1) if adjacent else (i, i + h)
    a, b = y[..., ia], y[..., ib]
    out, size = y.clone(), y.abs()
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = (a * c).abs() + (b * s).abs()
    size[..., ib] = (b * c).abs() + (a * s).abs()
    return out, size


def codes(y):
    """(values, scales) of fp32 heads [tokens, heads, d] in groups of 32."""
    n, h, d = y.shape
    g = y.reshape(n, h, d // 32, 32)
    top = g.abs().amax(3)
    alpha = (top / 6).clamp(min=2.0 ** -126).to(torch.bfloat16)
    mids = ((LEVELS[1:] + LEVELS[:-1]) / 2).to(y.device)
    v = LEVELS.to(y.device)[torch.bucketize((g.double() / alpha.double()[..., None]).abs(), mids, right=True)]
    v = torch.where(g < 0, -v, v)
    dead = ~torch.isfinite(top)
    alpha = torch.where(dead, float("nan"), alpha)
    return torch.where(dead[..., None], 0.0, v).reshape(n, h, d), alpha


def attend(q, k, v, last, scale):
    """One sequence in 64 bits: q [n, heads, d], k, v [m, kv heads, d], row i sees keys up to last[i].
    Returns (o, size, score, mass): size = sum p |v| / sum p, score = the largest scale sum |q k| of a row,
    mass = sum |v| over the keys that a row sees."""
    n, heads, d = q.shape
    m, kv = k.shape[:2]
    q = q.double().reshape(n, kv, heads // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
    k, v = k.double().permute(1, 2, 0).contiguous(), v.double().permute(1, 0, 2).contiguous()
    sees = torch.arange(m, device=q.device) <= last[:, None].to(q.device)
    sees = sees.repeat(heads // kv, 1)
    x = torch.where(sees, torch.matmul(q, k) * scale, -float("inf"))
    size = torch.where(sees, torch.matmul(q.abs(), k.abs()) * scale, 0.0).amax(2) if m else q.new_zeros(q.shape[:2])
    top = x.amax(2, keepdim=True) if m else x.sum(2, keepdim=True)
    p = torch.where(sees, torch.exp(x - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
    total = p.sum(2, keepdim=True)
    none = ~sees.any(1)[None, :, None]

    def back(t):
        return t.reshape(kv, heads // kv, n, t.shape[2]).permute(2, 0, 1, 3).reshape(n, heads, t.shape[2])

    o = torch.where(none, 0.0, torch.matmul(p, v) / total)
    s = torch.where(none, 0.0, torch.matmul(p, v.abs()) / total)
    return back(o), back(s), back(size[..., None]), back(torch.matmul(sees.double(), v.abs()))


def check(got, o, size, score, mass, keys, d, p_round, p_step=0.0):
    """fp32 scores of d products (error at most (d + 4) u of their magnitudes' sum, and twice that of a
    term's weight, since the maximum moves too), sums of `keys` terms, one rounding of each weighted
    probability to p_round, one of the output.  Probabilities whose type has a smallest step are off by half
    of it too, p_step, where the largest is 1 or more (and so is their sum)."""
    rel = p_round + 2 * (d + 4) * U * score + (keys + 8) * U
    u, step = ROUND[got.dtype], STEP[got.dtype]
    off = (got.double() - o).abs()
    work = rel * size + p_step * mass
    allowed = work + u * (o.abs() + work) + step
    assert bool((off <= allowed).all()), float((off / allowed.clamp(min=1e-300)).nan_to_num(nan=1e30).max())
