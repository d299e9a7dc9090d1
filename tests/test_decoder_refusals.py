"""The decoder operators' C entry points refuse bad arguments before any launch (no GPU)."""
import ctypes
import os

import pytest

from conftest import ROOT

LIB = os.path.join(ROOT, "paper_2109_03513_amd", "libesb.so")
INVALID, UNSUPPORTED, WORKSPACE = -1, -4, -6
F32, BF16, F16, E4M3 = range(4)
FAKE = ctypes.c_void_p(0x1000)      # never dereferenced
ODD = ctypes.c_void_p(0x1001)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(LIB):
        from paper_2109_03513_amd import build
        build.build()
    from paper_2109_03513_amd import esb
    return esb.lib()


def norm(L, x=FAKE, ldx=64, r=None, ldr=0, t=BF16, rows=4, d=64, w=FAKE, eps=1e-5, s=None, lds=0, y=FAKE,
         ldy=64, y8=None, ld8=0, scale=None):
    return L.esb_rmsnorm(x, ldx, r, ldr, t, rows, d, w, eps, s, lds, y, ldy, y8, ld8, scale, None)


def gated(L, g=FAKE, ldg=64, u=FAKE, ldu=64, t=BF16, rows=4, d=64, y=FAKE, ldy=64, y8=None, ld8=0, scale=None):
    return L.esb_swiglu(g, ldg, u, ldu, t, rows, d, y, ldy, y8, ld8, scale, None)


def test_rows(L):
    nan = float("nan")
    for bad in (dict(ldx=63), dict(t=E4M3), dict(t=7), dict(t=-1), dict(rows=-1), dict(d=-1), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=nan), dict(eps=float("inf")), dict(y=None), dict(ldy=63),
                dict(r=FAKE, ldr=63), dict(s=FAKE, lds=63), dict(y8=FAKE, ld8=64), dict(x=None),
                dict(y8=FAKE, ld8=63, scale=FAKE), dict(x=ODD), dict(y=ODD), dict(w=ODD),
                dict(y8=FAKE, ld8=64, scale=ODD), dict(s=ODD, lds=64), dict(r=ODD, ldr=64)):
        assert norm(L, **bad) == INVALID, bad
    assert norm(L, d=65537, ldx=65537, ldy=65537) == UNSUPPORTED
    assert norm(L, d=1 << 40, ldx=1 << 40, ldy=1 << 40) == UNSUPPORTED
    assert norm(L, rows=0, x=None) == 0 and norm(L, d=0, x=None) == 0
    for bad in (dict(ldg=63), dict(ldu=63), dict(u=None), dict(g=None), dict(t=E4M3), dict(rows=-1), dict(y=None),
                dict(y8=FAKE, ld8=64), dict(g=ODD), dict(u=ODD), dict(d=-5)):
        assert gated(L, **bad) == INVALID, bad
    assert gated(L, d=65537, ldg=65537, ldu=65537, ldy=65537) == UNSUPPORTED
    assert gated(L, rows=0, g=None, u=None) == 0


def test_weights(L):
    size = L.esb_w4_size
    assert size(32, 128, 128) == 2 * 1024 + 64
    assert size(33, 129, 32) == 2 * 3 * (1024 + 2 * 64)
    assert size(1, 65, 128) == 2 * 1024 + 64 and size(1, 1, 128) == 1024 + 64
    assert size(0, 128, 128) == 0 and size(16, 0, 128) == 0
    assert size(-1, 128, 128) == 0 and size(16, -1, 128) == 0 and size(16, 128, 16) == 0
    assert size((1 << 31) - 1, 1, 128) == 0 and size(1 << 26, 1 << 20, 128) == 0
    assert size(32, (1 << 30) + 1, 128) == 0 and size(32, 1 << 30, 128) > 1 << 34
    need = size(40, 200, 64)
    q = L.esb_w4_quantize

    def quant(w=FAKE, ldw=200, t=F32, N=40, K=200, g=64, f=FAKE, n=4, w4=FAKE, b=need):
        return q(w, ldw, t, N, K, g, f, n, w4, b, None)

    for bad in (dict(ldw=199), dict(t=E4M3), dict(N=-1), dict(K=-1), dict(g=65), dict(n=0), dict(n=65),
                dict(f=None), dict(w=None), dict(w4=None), dict(w4=ctypes.c_void_p(0x1008)), dict(w=ODD),
                dict(f=ODD)):
        assert quant(**bad) == INVALID, bad
    assert quant(b=need - 1) == WORKSPACE
    assert quant(N=(1 << 31) - 1) == UNSUPPORTED
    assert quant(N=0, w=None, w4=None, b=0) == 0
    p = L.esb_w4_pack
    assert p(FAKE, 199, FAKE, 4, 40, 200, 64, FAKE, need, None) == INVALID
    assert p(FAKE, 200, FAKE, 3, 40, 200, 64, FAKE, need, None) == INVALID
    assert p(FAKE, 200, ODD, 4, 40, 200, 64, FAKE, need, None) == INVALID
    assert p(None, 200, FAKE, 4, 40, 200, 64, FAKE, need, None) == INVALID
    assert p(FAKE, 200, FAKE, 4, 40, 200, 64, FAKE, need - 1, None) == WORKSPACE
    u = L.esb_w4_unpack
    assert u(FAKE, 40, 200, 64, None, 0, None, 0, None) == INVALID
    assert u(FAKE, 40, 200, 64, FAKE, 199, None, 0, None) == INVALID
    assert u(FAKE, 40, 200, 64, None, 0, FAKE, 3, None) == INVALID
    assert u(None, 40, 200, 64, FAKE, 200, None, 0, None) == INVALID
    assert u(FAKE, 40, 200, 33, FAKE, 200, None, 0, None) == INVALID


def test_products(L):
    def gemm(M=3, N=40, K=200, g=64, x=FAKE, ldx=200, t=BF16, s=None, w4=FAKE, y=FAKE, ldy=40, yt=BF16,
             ws=None, wb=0):
        return L.esb_w4_gemm(M, N, K, g, x, ldx, t, s, w4, y, ldy, yt, ws, wb, None)

    assert gemm(t=F32) == UNSUPPORTED
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(g=0), dict(ldx=199), dict(ldy=39), dict(t=4),
                dict(yt=E4M3), dict(x=None), dict(w4=None), dict(y=None), dict(x=ODD), dict(y=ODD), dict(s=ODD),
                dict(w4=ctypes.c_void_p(0x1004)), dict(ws=ctypes.c_void_p(0x1020), wb=1 << 30)):
        assert gemm(**bad) == INVALID, bad
    assert gemm(N=(1 << 31) - 1, ldy=1 << 40) == UNSUPPORTED
    assert gemm(M=0, x=None, y=None) == 0 and gemm(N=0, y=None) == 0
    size = L.esb_w4_gemm_workspace_size
    need = size(64, 512, 9216, 128, BF16, BF16)
    assert need > 0 and need % (64 * 512 * 4) == 0           # whole sets of fp32 sums
    big = dict(M=64, N=512, K=9216, g=128, ldx=9216, ldy=512, ws=FAKE)
    assert gemm(**big, wb=need - 1) == WORKSPACE
    assert size(1, 4096, 4096, 128, BF16, BF16) == 0 and size(4096, 18432, 4096, 128, E4M3, BF16) == 0
    assert size(2000, 4000, 4001, 64, BF16, BF16) >= 2000 * 4001 * 2       # rows to be aligned
    assert size(64, 4096, 4096, 100, BF16, BF16) == 0 and size(64, 4096, 4096, 128, F32, BF16) == 0


def test_host_weights(L):
    """Packed weights on the host are refused before anything is launched on their addresses."""
    import torch
    from paper_2109_03513_amd import esb
    w4 = torch.zeros(L.esb_w4_size(32, 64, 32), dtype=torch.uint8)
    with pytest.raises(TypeError):
        esb.esb_w4_unpack(w4, 32, 64, 32)
    with pytest.raises(TypeError):
        esb.esb_w4_unpack(w4.numpy(), 32, 64, 32)


def test_text_of_what_is_not_supported(L):
    """One status for the products of codes and the decoder operators: its text names both reasons."""
    text = L.esb_strerror(UNSUPPORTED)
    assert b"decoded integers exceed the split int8 range" in text and b"type or size" in text
