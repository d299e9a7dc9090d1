"""The C entry points of a decoder's attention refuse bad arguments before any launch (no GPU)."""
import ctypes
import os

import pytest
import torch

from conftest import ROOT

LIB = os.path.join(ROOT, "paper_2109_03513_amd", "libesb.so")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -4, -6
F32, BF16, F16, E4M3 = range(4)
FAKE, ODD, OTHER = 0x1000, 0x1001, 0x9000      # never dereferenced


@pytest.fixture(scope="module")
def esb():
    if not os.path.exists(LIB):
        from paper_2109_03513_amd import build
        build.build()
    from paper_2109_03513_amd import esb
    esb.lib()
    return esb


def ref(s):
    return None if s is None else ctypes.byref(s)


def heads(esb, n=4, d=64, data=FAKE, token=None, head=None):
    return esb.Heads(data, n * d if token is None else token, d if head is None else head, n)


def rotation(esb, **kw):
    r = dict(table=FAKE, rows=100, rot=64, adjacent=0, positions=FAKE)
    r.update(kw)
    return esb.Rotation(*r.values())


def rope(esb, q=0, k=0, t=BF16, tokens=3, d=64, qw=None, kw=None, eps=0.0, r=0, qo=0, ko=0):
    h = lambda v: heads(esb, d=d) if v == 0 else v  # noqa: E731
    r = rotation(esb) if r == 0 else r
    return esb.lib().esb_rope(ref(h(q)), ref(h(k)), t, tokens, d, qw, kw, eps, ref(r), ref(h(qo)), ref(h(ko)), None)


def test_rope(esb):
    nan, inf = float("nan"), float("inf")
    H = lambda **kw: heads(esb, **kw)  # noqa: E731
    R = lambda **kw: rotation(esb, **kw)  # noqa: E731
    for bad in (dict(t=E4M3), dict(t=9), dict(tokens=-1), dict(d=0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf),
                dict(qw=FAKE), dict(qw=ODD, eps=1e-5), dict(kw=ODD, eps=1e-5), dict(q=None), dict(ko=None),
                dict(q=None, k=None, qo=None, ko=None), dict(q=H(data=None)), dict(q=H(data=ODD)), dict(q=H(n=0)),
                dict(q=H(token=-1)), dict(k=H(head=-64)), dict(qo=H(n=3)), dict(qo=H(token=0)), dict(qo=H(head=63)),
                dict(qo=H(head=0)), dict(qo=H(token=255)), dict(ko=H(token=64)), dict(ko=H(token=64, head=191)),
                dict(r=R(rot=63)), dict(r=R(rot=66)), dict(r=R(rot=-2)), dict(r=R(rows=-1)),
                dict(r=R(table=None)), dict(r=R(positions=None)), dict(r=R(table=ODD)), dict(r=R(positions=ODD))):
        assert rope(esb, **bad) == INVALID, bad
    assert rope(esb, d=513, r=None) == UNSUPPORTED
    assert rope(esb, q=H(n=5000), qo=H(n=5000)) == UNSUPPORTED
    empty = H(data=None)
    assert rope(esb, tokens=0, q=empty, k=empty, qo=empty, ko=empty) == OK
    assert rope(esb, tokens=0, q=None, qo=None) == OK


def kv4(esb, **kw):
    c = dict(data=FAKE, pages=9, page=16, heads=4, d=64)
    c.update(kw)
    return esb.Kv4(*c.values())


def test_cache(esb):
    size = esb.lib().esb_kv4_page_size
    assert size(16, 4, 64) == 16 * 4 * 72 and size(64, 8, 128) == 64 * 8 * 144 and size(16, 1, 256) == 16 * 288
    for bad in ((8, 4, 64), (24, 4, 64), (8192, 4, 64), (0, 4, 64), (-16, 4, 64), (16, 0, 64), (16, 4, 48), (16, 4, 288),
                (16, 4, 0), (16, 5000, 64)):
        assert size(*bad) == 0, bad

    def append(q=None, k=0, v=0, t=BF16, tokens=3, qw=None, kw=None, eps=0.0, r=None, slots=FAKE, c=0, qo=None):
        h = lambda x: heads(esb) if x == 0 else x  # noqa: E731
        c = kv4(esb) if c == 0 else c
        return esb.lib().esb_kv4_append(ref(q), ref(h(k)), ref(h(v)), t, tokens, qw, kw, eps, ref(r), slots, ref(c),
                                        ref(qo), None)

    H = lambda **kw: heads(esb, **kw)  # noqa: E731
    for bad in (dict(k=None), dict(v=None), dict(c=None), dict(t=E4M3), dict(tokens=-1), dict(slots=None),
                dict(slots=FAKE + 4), dict(k=H(n=3)), dict(v=H(n=5)), dict(v=H(data=ODD)), dict(kw=FAKE),
                dict(q=H()), dict(qo=H()), dict(qw=FAKE, eps=1e-5), dict(q=H(), qo=H(n=3)),
                dict(c=kv4(esb, data=None)), dict(c=kv4(esb, data=FAKE + 8)), dict(c=kv4(esb, pages=-1)),
                dict(c=kv4(esb, page=0)), dict(r=rotation(esb, rot=128))):
        assert append(**bad) == INVALID, bad
    for bad in (dict(page=24), dict(page=8), dict(d=72), dict(d=512), dict(pages=1 << 31)):
        assert append(c=kv4(esb, **bad)) == UNSUPPORTED, bad
    assert append(tokens=0, k=H(data=None), v=H(data=None), slots=None) == OK
    L = esb.lib()

    def pack(k=FAKE, ka=FAKE, v=FAKE, va=FAKE, n=3, slots=FAKE):
        return L.esb_kv4_pack(k, ka, v, va, n, slots, ref(kv4(esb)), None)

    for bad in (dict(k=None), dict(ka=None), dict(v=None), dict(va=None), dict(ka=ODD), dict(va=ODD), dict(n=-1),
                dict(slots=None), dict(slots=FAKE + 1)):
        assert pack(**bad) == INVALID, bad
    assert pack(n=0, k=None) == OK

    def unpack(k=FAKE, ka=FAKE, v=FAKE, va=FAKE, n=3, slots=FAKE):
        return L.esb_kv4_unpack(ref(kv4(esb)), n, slots, k, ka, v, va, None)

    for bad in (dict(k=None, ka=None, v=None, va=None), dict(ka=ODD), dict(va=ODD), dict(n=-1), dict(slots=None)):
        assert unpack(**bad) == INVALID, bad
    assert unpack(n=0, slots=None) == OK


def test_cache_attention(esb):
    L = esb.lib()
    size = L.esb_kv4_attention_workspace_size
    need = size(3, 8, 64, 4, 3, 0, 640, 16)
    assert need > 0 and size(3, 8, 64, 4, 3, 0, 0, 16) == 0
    for bad in ((-1, 8, 64, 4, 3, 0, 64, 16), (3, 7, 64, 4, 3, 0, 64, 16), (3, 8, 48, 4, 3, 0, 64, 16),
                (3, 8, 64, 4, -3, 0, 64, 16), (3, 8, 64, 4, 3, 0, -1, 16), (3, 8, 64, 4, 3, 0, 1 << 40, 16),
                (3, 8, 64, 4, 3, 0, 64, 20)):
        assert size(*bad) == 0, bad

    def attend(q=0, t=BF16, tokens=3, c=0, seqs=3, starts=None, lengths=FAKE, pages=FAKE, pitch=640, columns=640,
               scale=0.1, o=0, ws=FAKE, wb=need):
        q = heads(esb, n=8) if q == 0 else q
        o = heads(esb, n=8, data=OTHER) if o == 0 else o
        c = kv4(esb) if c == 0 else c
        return L.esb_kv4_attention(ref(q), t, tokens, ref(c), seqs, starts, lengths, pages, pitch, columns, scale,
                                   ref(o), ws, wb, None)

    H = lambda **kw: heads(esb, **kw)  # noqa: E731
    for bad in (dict(q=None), dict(o=None), dict(c=None), dict(t=E4M3), dict(tokens=-1), dict(tokens=2), dict(seqs=-1),
                dict(lengths=None), dict(pages=None), dict(pitch=639), dict(columns=-1), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(o=H(n=8)),
                dict(q=H(n=6), o=H(n=6, data=OTHER)), dict(o=H(n=4, data=OTHER)), dict(starts=ODD), dict(lengths=ODD),
                dict(pages=ODD), dict(ws=FAKE + 16), dict(q=H(n=8, data=ODD)), dict(o=H(n=8, data=OTHER, token=0)),
                dict(c=kv4(esb, pages=0, data=None))):
        assert attend(**bad) == INVALID, bad
    assert attend(t=F32) == UNSUPPORTED
    assert attend(columns=1 << 28, pitch=1 << 28) == UNSUPPORTED
    assert attend(columns=1 << 24, pitch=1 << 24, tokens=1 << 18, seqs=1 << 18) == UNSUPPORTED
    assert attend(tokens=1 << 28, seqs=1 << 28) == UNSUPPORTED
    assert attend(ws=None) == WORKSPACE and attend(wb=need - 1) == WORKSPACE
    none = H(n=8, data=None)
    assert attend(tokens=0, seqs=0, q=none, o=none, lengths=None, pages=None, ws=None, wb=0) == OK


def test_attention(esb):
    L = esb.lib()

    def attend(q=0, k=0, v=0, t=BF16, nq=3, nk=3, d=64, seqs=2, qs=FAKE, ks=None, causal=1, scale=0.1, o=0):
        h = lambda x, n, **kw: heads(esb, n=n, **kw) if x == 0 else x  # noqa: E731
        return L.esb_attention(ref(h(q, 8)), ref(h(k, 4)), ref(h(v, 4)), t, nq, nk, d, seqs, qs, ks, causal, scale,
                               ref(h(o, 8, data=OTHER)), None)

    H = lambda **kw: heads(esb, **kw)  # noqa: E731
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(t=E4M3), dict(nq=-1), dict(nk=-1), dict(d=0),
                dict(seqs=-1), dict(qs=None), dict(qs=ODD), dict(ks=ODD), dict(nk=4), dict(scale=0.0),
                dict(scale=float("nan")), dict(k=H(n=3), v=H(n=3)), dict(v=H(n=2)), dict(o=H(n=4, data=OTHER)),
                dict(o=H(n=8)), dict(k=H(data=None)), dict(q=H(n=8, data=ODD)), dict(o=H(n=8, data=OTHER, head=0)), dict(scale=3e38),
                dict(k=H(data=OTHER)), dict(v=H(data=OTHER))):
        assert attend(**bad) == INVALID, bad
    assert attend(t=F32) == UNSUPPORTED
    assert attend(d=60) == UNSUPPORTED and attend(d=264) == UNSUPPORTED
    assert attend(nq=1 << 29, nk=1 << 29) == UNSUPPORTED
    none = H(n=8, data=None)
    assert attend(nq=0, nk=0, q=none, o=none, k=H(data=None), v=H(data=None), qs=None) == OK


def test_host_tensors(esb):
    """The binding refuses tensors on the host before their addresses go anywhere."""
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    n = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        esb.esb_rope(x)
    with pytest.raises(TypeError):
        esb.esb_kv4_append(torch.zeros(2, 4608, dtype=torch.uint8), 16, x, x, n.long())
    with pytest.raises(TypeError):
        esb.esb_kv4_unpack(torch.zeros(2, 4608, dtype=torch.uint8), 16, 4, 64, n.long())
    with pytest.raises(TypeError):
        esb.esb_kv4_attention(x, torch.zeros(2, 4608, dtype=torch.uint8), 16, 4, n[:, None], n)
    with pytest.raises(TypeError):
        esb.esb_attention(x, x, x, n)


def test_attention_of_most_rows_and_keys(esb):
    """Rows and keys whose tiles would end past 32 bits: their indexes, and the loop over the keys, would wrap."""
    L = esb.lib()
    one = heads(esb, n=1, d=8)
    out = heads(esb, n=1, d=8, data=OTHER)
    most = (1 << 31) - 1

    def attend(nq, nk, seqs=1):
        return L.esb_attention(ref(one), ref(one), ref(one), BF16, nq, nk, 8, seqs, FAKE, FAKE, 1, 0.1, ref(out), None)

    for nk in (most, most - 64, most - 8191):
        assert attend(3, nk) == UNSUPPORTED, nk
    for nq in (most - 1, most - 100, most - 8191):
        assert attend(nq, 3) == UNSUPPORTED, nq
    # a group of heads counts each of them
    q, o = (heads(esb, n=64, d=8, data=x) for x in (FAKE, OTHER))
    assert L.esb_attention(ref(q), ref(one), ref(one), BF16, (1 << 25) - 2, 3, 8, 1, FAKE, FAKE, 1, 0.1, ref(o), None) == UNSUPPORTED
