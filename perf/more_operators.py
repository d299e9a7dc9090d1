"""Timed cases of a decoder's attention: the norm and rotation of query and key heads, the 4-bit
paged cache that keys and values are appended to, the attention that reads it, and the attention
over whole prompts.

    listed()             the named cases
    draw(rng)            one more case from the same ranges
    prepare(case, seed)  inputs and caches, on the GPU
    run(state)           one pass: plain torch in 32 bits, or (own) the library's entry points
    work(case)           bytes and operations the pass cannot do without
    exact(case, seed)    what run() returns, from the definitions in 64 bits

What the cache holds is returned as its unscaled values (exact in E4M3) and bf16 scales.
"""
import math
import random

import torch

own = False

EPS = 1e-6
GROUP = 32
TINY = 2.0 ** -126                 # the least scale: the smallest normal number
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]      # magnitudes of ESB(4,1) = E2M1


def listed():
    return [
        # the heads of one new token: the smallest call, all latency
        dict(name="rope_token", kind="rope", tokens=1, q_heads=32, kv_heads=8, d=128, rot=128,
             pairs="halves", norm=True, type="bf16"),
        # fp32 heads of odd numbers and length, the first half of each rotated in adjacent pairs
        dict(name="rope_ragged_f32", kind="rope", tokens=1999, q_heads=7, kv_heads=3, d=80, rot=40,
             pairs="adjacent", norm=False, type="f32"),
        # a prompt's heads
        dict(name="rope_prompt", kind="rope", tokens=4096, q_heads=32, kv_heads=8, d=128, rot=128,
             pairs="halves", norm=True, type="bf16"),
        # one token of each of a batch of decoding requests, anywhere in the cache, queries too
        dict(name="append_batch", kind="append", tokens=64, q_heads=32, kv_heads=8, d=128, rot=128,
             pairs="halves", norm=True, type="bf16", page=64, queries=True, decode=True),
        # a ragged prompt of short heads, small pages
        dict(name="append_ragged_f16", kind="append", tokens=777, q_heads=6, kv_heads=3, d=96,
             rot=48, pairs="adjacent", norm=False, type="f16", page=16, queries=False,
             decode=False),
        # a prompt's keys and values
        dict(name="append_prompt", kind="append", tokens=4096, q_heads=32, kv_heads=8, d=128,
             rot=128, pairs="halves", norm=True, type="bf16", page=64, queries=False,
             decode=False),
        # one request's next token after a long context
        dict(name="cache_token", kind="cache", seqs=1, new=1, longest=32768, q_heads=32, kv_heads=8,
             d=128, type="bf16", page=64, mix=1),
        # a batch of requests of different lengths, the next token of each
        dict(name="cache_batch", kind="cache", seqs=64, new=1, longest=8192, q_heads=32, kv_heads=8,
             d=128, type="bf16", page=64, mix=2),
        # several tokens a request (drafts to be verified), short heads, fp16, small pages
        dict(name="cache_drafts_f16", kind="cache", seqs=24, new=5, longest=3001, q_heads=14,
             kv_heads=2, d=64, type="f16", page=16, mix=3),
        # the next part of a long prompt, against what the cache holds of it
        dict(name="cache_part", kind="cache", seqs=2, new=512, longest=8192, q_heads=32, kv_heads=8,
             d=128, type="bf16", page=64, mix=4),
        # prompts of different lengths in one pack, fp16, short heads
        dict(name="prompt_pack_f16", kind="prompt", seqs=9, tokens=4001, before=0, q_heads=12,
             kv_heads=4, d=64, type="f16", causal=True, mix=5),
        # the largest: one long prompt
        dict(name="prompt_long", kind="prompt", seqs=1, tokens=8192, before=0, q_heads=32,
             kv_heads=8, d=128, type="bf16", causal=True, mix=6),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "cache", "cache", "cache", "prompt", "prompt"])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 7])
    if q_heads > 32:
        q_heads = 32
    case = dict(kind=kind, q_heads=q_heads, kv_heads=kv_heads)
    if kind in ("rope", "append"):
        d = rng.choice([64, 96, 128, 128, 256] if kind == "append" else [64, 80, 96, 128, 128, 256])
        case.update(tokens=_log(rng, 1, 4096), d=d, rot=rng.choice([d, d, d // 2]),
                    pairs=rng.choice(["halves", "adjacent"]), norm=rng.random() < 0.6,
                    type=rng.choice(["bf16", "bf16", "f16", "f32"]))
        if kind == "append":
            decode = case["tokens"] <= 256 and rng.random() < 0.5
            case.update(page=rng.choice([16, 32, 64, 128]), queries=rng.random() < 0.5,
                        decode=decode)
        return case
    case.update(type=rng.choice(["bf16", "bf16", "f16"]), mix=rng.randrange(1 << 20))
    if kind == "cache":
        seqs, new = _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 5, 64, 300, 512])
        longest = _log(rng, max(new, 16), 32768)
        while new > 1 and seqs * new > 1024:
            seqs = max(1, seqs // 2)
        if seqs * longest > 64 * 8192:
            longest = max(new, 64 * 8192 // seqs)
        case.update(seqs=seqs, new=new, longest=longest, d=rng.choice([64, 96, 128, 128, 256]),
                    page=rng.choice([16, 32, 64, 128]))
        if case["d"] == 256:
            case["longest"] = max(new, longest // 2)
        return case
    seqs, tokens = _log(rng, 1, 32), _log(rng, 32, 4096)
    case.update(seqs=min(seqs, tokens), tokens=tokens, before=rng.choice([0, 0, 0, _log(rng, 1, 512)]),
                d=rng.choice([64, 80, 96, 128, 128, 256]), causal=rng.random() < 0.8)
    if case["d"] == 256:
        case["tokens"] = max(case["seqs"], tokens // 2)
    return case


# ---- lengths --------------------------------------------------------------------------------


def _split(case):
    """Tokens of each packed sequence: at least one, `tokens` in all."""
    rng = random.Random(case["mix"])
    share = [rng.random() ** 2 + 0.02 for _ in range(case["seqs"])]
    lengths = [1 + int(s / sum(share) * (case["tokens"] - case["seqs"])) for s in share]
    lengths[0] += case["tokens"] - sum(lengths)
    return lengths


def _lengths(case):
    """(new tokens, cached tokens with them) of each sequence of a cache."""
    rng = random.Random(case["mix"])
    new = [case["new"] if case["new"] < 2 or i == 0 else rng.randint(1, case["new"])
           for i in range(case["seqs"])]
    kept = [case["longest"] if i == 0 else max(n, rng.randint(case["longest"] // 4, case["longest"]))
            for i, n in enumerate(new)]
    return new, kept


def _starts(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32,
                        device="cuda")


# ---- inputs ---------------------------------------------------------------------------------


def _qkv(g, tokens, q_heads, kv_heads, d, dtype):
    """Heads of q, k and v, the columns of one product's rows: a few channels of k are large."""
    n = q_heads + 2 * kv_heads
    x = torch.randn(tokens, n, d, generator=g, device="cuda")
    channel = torch.exp(0.4 * torch.randn(n, d, generator=g, device="cuda"))
    big = torch.rand(n, d, generator=g, device="cuda") < 0.01
    big[:q_heads] = big[q_heads + kv_heads:] = False
    x = (x * torch.where(big, 8 * channel, channel)).to(dtype)
    return x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]


def _table(rows, rot):
    """Cosines, then sines, of a position's angles: one row a position, from 64 bits."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([torch.cos(a), torch.sin(a)], 1).float()


def _codes(g, shape):
    """Magnitude index | sign << 3 of normal values under a group's scale."""
    p = (torch.arange(128, dtype=torch.float64, device="cuda") + 0.5) / 128
    v = 2.5 * math.sqrt(2) * torch.erfinv(p)
    mids = (torch.tensor(LEVELS[1:], device="cuda") + torch.tensor(LEVELS[:-1], device="cuda")) / 2
    m = torch.bucketize(v.float(), mids).to(torch.uint8)
    m = torch.cat([m, m | 8])
    return m[torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8).int()]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, d, s = case["kind"], case["d"], {}
    t = TYPES[case["type"]]
    if kind in ("rope", "append"):
        n = case["tokens"]
        s["q"], s["k"], s["v"] = _qkv(g, n, case["q_heads"], case["kv_heads"], d, t)
        s["table"] = _table(32768 if n < 512 else 8192, case["rot"])
        if kind == "rope" and n < 512 or kind == "append" and case["decode"]:
            s["positions"] = torch.randint(0, 32768 if n < 512 else 8192, (n,), generator=g,
                                           device="cuda", dtype=torch.int32)
        else:
            s["positions"] = torch.arange(n, device="cuda", dtype=torch.int32)
        for w in ("q_w", "k_w"):
            s[w] = 1 + 0.2 * torch.randn(d, generator=g, device="cuda") if case["norm"] else None
        if kind == "append":
            page = case["page"]
            pages = 2 * (n // page + 1) if not case["decode"] else 4 * n
            order = torch.randperm(pages, generator=g, device="cuda")
            i = torch.arange(n, device="cuda")
            if case["decode"]:       # a page of its own for every token, anywhere in it
                s["slots"] = order[i] * page + torch.randint(0, page, (n,), generator=g, device="cuda")
            else:
                s["slots"] = order[i // page] * page + i % page
            s["pages"] = pages
        return s
    if kind == "cache":
        new, kept = _lengths(case)
        page, heads = case["page"], case["kv_heads"]
        columns = -(-max(kept) // page)
        total = sum(-(-k // page) for k in kept)
        order = torch.randperm(total, generator=g, device="cuda").int()
        pages, at = torch.zeros(case["seqs"], columns, dtype=torch.int32, device="cuda"), 0
        for i, k in enumerate(kept):
            c = -(-k // page)
            pages[i, :c] = order[at:at + c]
            at += c
        s.update(pages=pages, total=total, lengths=torch.tensor(kept, dtype=torch.int32, device="cuda"),
                 starts=_starts(new) if case["new"] > 1 else None)
        for x in ("k", "v"):
            s[x] = _codes(g, (total * page, heads, d))
            s[x + "_alpha"] = (0.4 * torch.exp(0.3 * torch.randn(
                total * page, heads, d // GROUP, generator=g, device="cuda"))).to(torch.bfloat16)
        s["q"] = _qkv(g, sum(new), case["q_heads"], heads, d, t)[0]
        return s
    lengths = _split(case)
    before = case["before"]
    s["q"] = _qkv(g, case["tokens"], case["q_heads"], case["kv_heads"], d, t)[0]
    s["k"], s["v"] = _qkv(g, case["tokens"] + before * case["seqs"], 0, case["kv_heads"], d, t)[1:]
    s["q_starts"] = _starts(lengths)
    s["k_starts"] = _starts([n + before for n in lengths])
    return s


def _index(starts, width):
    """Rows of a pack as a padded batch: [sequences, width] indexes and which of them are there."""
    at = starts[:-1, None].long() + torch.arange(width, device="cuda")
    there = at < starts[1:, None]
    return torch.where(there, at, 0), there


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind, d = case["kind"], case["d"]
    if kind == "append":
        heads, page, slots = case["kv_heads"], case["page"], s["pages"] * case["page"]
        if own:
            from paper_2109_03513_amd import esb
            s["cache"] = torch.zeros(s["pages"], esb.esb_kv4_page_size(page, heads, d),
                                     dtype=torch.uint8, device="cuda")
        else:
            for x in ("k", "v"):
                s[x + "_cache"] = torch.zeros(slots, heads, d // 2, dtype=torch.uint8, device="cuda")
                s[x + "_scales"] = torch.zeros(slots, heads, d // GROUP, dtype=torch.bfloat16,
                                               device="cuda")
    elif kind == "cache":
        # the cache as each side keeps it: the library's pages, or two codes to a byte
        codes = s.pop("k"), s.pop("v")
        if own:
            from paper_2109_03513_amd import esb
            page, heads = case["page"], case["kv_heads"]
            s["cache"] = torch.zeros(s["total"], esb.esb_kv4_page_size(page, heads, d),
                                     dtype=torch.uint8, device="cuda")
            slots = torch.arange(s["total"] * page, device="cuda")
            # ESB(4,1) codes: 1, 1.5, 2, 3, 4, 6, 0, 0.5 are 0 .. 7
            k, v = (((c & 7) + 6) & 7 | (c & 8) for c in codes)
            esb.esb_kv4_pack(s["cache"], page, k, s.pop("k_alpha"), v, s.pop("v_alpha"), slots)
        else:
            s["k"], s["v"] = (c[..., 0::2] | (c[..., 1::2] << 4) for c in codes)
            new, kept = _lengths(case)
            s["width"], s["new"] = max(kept), max(new)
    elif kind == "prompt" and not own:
        lengths = _split(case)
        s["width"], s["k_width"] = max(lengths), max(lengths) + case["before"]
    return s


# ---- one pass -------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, case):
    from paper_2109_03513_amd import esb
    kind = case["kind"]
    if kind in ("rope", "append"):
        how = dict(eps=EPS if case["norm"] else 0.0, k_w=s["k_w"],
                   adjacent=case["pairs"] == "adjacent")
    if kind == "rope":
        q, k = esb.esb_rope(s["q"], s["k"], s["table"], s["positions"], q_w=s["q_w"], **how)
        return {"q": q, "k": k}
    if kind == "append":
        queries = dict(q=s["q"], q_w=s["q_w"]) if case["queries"] else {}
        q = esb.esb_kv4_append(s["cache"], case["page"], s["k"], s["v"], s["slots"], s["table"],
                               s["positions"], **queries, **how)
        k, k_alpha, v, v_alpha = esb.esb_kv4_unpack(s["cache"], case["page"], case["kv_heads"],
                                                    case["d"], s["slots"])
        return {"q": q, "k": k, "k_alpha": k_alpha, "v": v, "v_alpha": v_alpha}
    if kind == "cache":
        return {"o": esb.esb_kv4_attention(s["q"], s["cache"], case["page"], case["kv_heads"],
                                           s["pages"], s["lengths"], starts=s["starts"])}
    return {"o": esb.esb_attention(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"],
                                   causal=case["causal"])}


def _turn(x, w, s, case):
    """Norm and rotation of heads, in x's precision."""
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * w
    rot = case["rot"]
    row = s["table"][s["positions"].long()][:, None].to(x.dtype)
    c, n = row[..., :rot // 2], row[..., rot // 2:]
    if case["pairs"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * n, b * c + a * n], 2)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * n, b * c + a * n], 3).flatten(2)
    return torch.cat([turned, x[..., rot:]], 2)


def _four_bits(y):
    """Codes (magnitude index | sign << 3) and scales of fp32 heads, values next to a border in 64 bits."""
    y = y.unflatten(2, (-1, GROUP))
    alpha = (y.abs().amax(3) / 6).clamp(min=TINY).to(torch.bfloat16)
    a = (y.double() / alpha.double()[..., None]).abs()
    m = sum((a >= (lo + hi) / 2).to(torch.uint8) for lo, hi in zip(LEVELS, LEVELS[1:]))
    return (m | ((y < 0) & (m > 0)).to(torch.uint8) << 3).flatten(2), alpha


def _values():
    v = torch.tensor(LEVELS, device="cuda")
    return torch.cat([v, -v])


def _unpacked(c):
    return _values()[torch.stack([c & 15, c >> 4], -1).flatten(-2).int()]


def _attend(q, k, v, sees, scale):
    """q [b, n, heads, d], k and v [b, m, kv heads, d], sees [b, n, m], in 32 bits."""
    b, n, heads, d = q.shape
    m, kv = k.shape[1:3]
    group = heads // kv
    q = q.unflatten(2, (kv, group)).permute(0, 2, 3, 1, 4).reshape(b * kv, group * n, d)
    k = k.permute(0, 2, 3, 1).reshape(b * kv, d, m)
    v = v.permute(0, 2, 1, 3).reshape(b * kv, m, d)
    x = torch.matmul(q, k).mul_(scale).view(b, kv * group, n, m)
    sees = sees[:, None]
    x = x.masked_fill_(~sees, -math.inf)
    top = x.amax(3, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = x.sum(3, keepdim=True)
    o = torch.matmul(x.view(b * kv, group * n, m), v).view(b, kv * group, n, d)
    o = torch.where(total > 0, o / total, 0)
    return o.transpose(1, 2)


def _run_plain(s, case):
    kind, d = case["kind"], case["d"]
    if kind == "rope":
        t = s["q"].dtype
        return {"q": _turn(s["q"].float(), s["q_w"], s, case).to(t),
                "k": _turn(s["k"].float(), s["k_w"], s, case).to(t)}
    if kind == "append":
        q = None
        if case["queries"]:
            q = _turn(s["q"].float(), s["q_w"], s, case).to(s["q"].dtype)
        out = {"q": q}
        # borders between codes: the heads in 64 bits, rounded once to 32
        y = {"k": _turn(s["k"].double(), s["k_w"], s, case).float(), "v": s["v"].float()}
        for x in ("k", "v"):
            codes, alpha = _four_bits(y[x])
            s[x + "_cache"][s["slots"]] = codes[..., 0::2] | (codes[..., 1::2] << 4)
            s[x + "_scales"][s["slots"]] = alpha
            out[x] = _unpacked(s[x + "_cache"][s["slots"]]).to(torch.float8_e4m3fn)
            out[x + "_alpha"] = s[x + "_scales"][s["slots"]]
        return out
    if kind == "cache":
        j = torch.arange(s["width"], device="cuda")
        slots = s["pages"][:, j // case["page"]].long() * case["page"] + j % case["page"]
        k, v = (_unpacked(s[x][slots]).unflatten(3, (-1, GROUP)).mul_(
            s[x + "_alpha"][slots].float()[..., None]).flatten(3) for x in ("k", "v"))
        i = torch.arange(s["new"], device="cuda")
        if s["starts"] is None:
            q, there, new = s["q"][:, None], None, torch.ones_like(s["lengths"])
        else:
            at, there = _index(s["starts"], s["new"])
            q, new = s["q"][at], s["starts"].diff()
        last = (s["lengths"] - new)[:, None] + i                     # the last key a query sees
        sees = (j <= last[..., None]) & (j < s["lengths"][:, None, None])
        o = _attend(q.float(), k, v, sees, d ** -0.5)
        return {"o": (o[:, 0] if there is None else o[there]).to(s["q"].dtype)}
    at, there = _index(s["q_starts"], s["width"])
    k_at, k_there = _index(s["k_starts"], s["k_width"])
    sees = k_there[:, None].expand(-1, s["width"], -1)
    if case["causal"]:
        i, j = torch.arange(s["width"], device="cuda"), torch.arange(s["k_width"], device="cuda")
        sees = sees & (j <= i[:, None] + case["before"])
    o = _attend(s["q"][at].float(), s["k"][k_at].float(), s["v"][k_at].float(), sees, d ** -0.5)
    return {"o": o[there].to(s["q"].dtype)}


# ---- what a pass needs ----------------------------------------------------------------------


def work(case):
    kind, d = case["kind"], case["d"]
    heads, kv = case["q_heads"], case["kv_heads"]
    t = SIZE[case["type"]]
    if kind in ("rope", "append"):
        n = case["tokens"]
        per = case["rot"] * 4 + 4                    # a row of the table, and which
        if kind == "rope":
            return {"bytes": n * ((heads + kv) * d * 2 * t + per), "flops": n * (heads + kv) * d * 7}
        turned = (heads if case["queries"] else 0) * d * 2 * t
        # keys and values in, their codes and scales out, and what the pass returns of them
        cached = 2 * kv * (d * t + d / 2 + 2 * d / GROUP + d + 2 * d / GROUP)
        return {"bytes": n * (turned + cached + per + 8), "flops": n * (heads + 2 * kv) * d * 9}
    if kind == "cache":
        new, kept = _lengths(case)
        pairs = sum(n * k - n * (n - 1) // 2 for n, k in zip(new, kept))
        cached = sum(kept) * kv * 2 * (d / 2 + 2 * d / GROUP)
        return {"bytes": cached + sum(new) * heads * d * 2 * t, "flops": 4 * pairs * heads * d}
    lengths = _split(case)
    before = case["before"]
    pairs = sum(n * (n + before) - (n * (n - 1) // 2 if case["causal"] else 0) for n in lengths)
    keys = case["tokens"] + case["seqs"] * before
    return {"bytes": t * d * (2 * case["tokens"] * heads + 2 * keys * kv),
            "flops": 4 * pairs * heads * d}


# ---- the definitions in 64 bits -------------------------------------------------------------


def _exact_turn(x, w, s, case):
    z, rot = x.double(), case["rot"]
    if case["norm"]:
        z = z / torch.sqrt((z * z).sum(-1, keepdim=True) / case["d"] + EPS) * w.double()
    angle = s["table"].double()[s["positions"].long()]
    turn = torch.complex(angle[:, :rot // 2], angle[:, rot // 2:])[:, None]
    out = z.clone()
    if case["pairs"] == "halves":
        u = torch.complex(z[..., :rot // 2], z[..., rot // 2:rot].contiguous()) * turn
        out[..., :rot // 2], out[..., rot // 2:rot] = u.real, u.imag
    else:
        u = torch.complex(z[..., 0:rot:2].contiguous(), z[..., 1:rot:2].contiguous()) * turn
        out[..., 0:rot:2], out[..., 1:rot:2] = u.real, u.imag
    return out


def _exact_codes(y):
    """(values, scales) of heads, whose values are fp32 numbers."""
    y = y.float()
    levels = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    mids = (levels[1:] + levels[:-1]) / 2
    blocks = y.reshape(y.shape[0], y.shape[1], -1, GROUP)
    top = torch.linalg.vector_norm(blocks, float("inf"), dim=3)
    alpha = torch.maximum(top / 6, torch.full_like(top, TINY)).to(torch.bfloat16).double()
    u = blocks.double() / alpha[..., None]
    v = torch.copysign(levels[torch.bucketize(u.abs(), mids, right=True)], u)
    return v.reshape(y.shape), alpha


def _exact_one(q, k, v, before, causal):
    """One sequence: q [n, heads, d], k and v [m, kv heads, d]; row i sees keys up to i + before."""
    n, heads, d = q.shape
    m, group = k.shape[0], heads // k.shape[1]
    o = torch.empty(n, heads, d, dtype=torch.float64, device="cuda")
    hidden = torch.arange(m, device="cuda") > torch.arange(n, device="cuda")[:, None] + before
    for h in range(heads):
        x = torch.mm(q[:, h].double(), k[:, h // group].double().t()) / math.sqrt(d)
        if causal:
            x[hidden] = -math.inf
        o[:, h] = torch.mm(torch.softmax(x, 1), v[:, h // group].double())
    return o


def exact(case, seed):
    s = _inputs(case, seed)
    kind, d = case["kind"], case["d"]
    if kind == "rope":
        return {"q": _exact_turn(s["q"], s["q_w"], s, case), "k": _exact_turn(s["k"], s["k_w"], s, case)}
    if kind == "append":
        out = {"q": _exact_turn(s["q"], s["q_w"], s, case) if case["queries"] else None}
        out["k"], out["k_alpha"] = _exact_codes(_exact_turn(s["k"], s["k_w"], s, case))
        out["v"], out["v_alpha"] = _exact_codes(s["v"].double())
        return out
    if kind == "cache":
        levels = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device="cuda")
        new, kept = _lengths(case)
        o, at, page = [], 0, case["page"]
        for i, (n, m) in enumerate(zip(new, kept)):
            where = s["pages"][i, :-(-m // page)].long()[:, None] * page
            where = (where + torch.arange(page, device="cuda")).flatten()[:m]
            k, v = (levels[s[x][where].int()] * s[x + "_alpha"][where].double().repeat_interleave(GROUP, 2)
                    for x in ("k", "v"))
            o.append(_exact_one(s["q"][at:at + n], k, v, m - n, True))
            at += n
        return {"o": torch.cat(o)}
    o, at, k_at = [], 0, 0
    for n in _split(case):
        m = n + case["before"]
        o.append(_exact_one(s["q"][at:at + n], s["k"][k_at:k_at + m], s["v"][k_at:k_at + m],
                            case["before"], case["causal"]))
        at, k_at = at + n, k_at + m
    return {"o": torch.cat(o)}
