"""Thin ctypes binding of libesb (include/esb.h), same entry-point names.

Argument marshalling only: every step of the hot path runs in the HIP kernels
of libesb.so.  PyTorch provides device memory and streams.  If libesb.so is
missing the import of any entry point raises; there is no fallback.
"""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libesb.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "esb.h")

ESB_OK = 0
ESB_E_INVALID = -1
ESB_E_OVERFLOW = -3
ESB_E_UNSUPPORTED = -4
ESB_E_HIP = -5
ESB_E_WORKSPACE = -6
ESB_E_SCRATCH = -7
ESB_DDA_NOALLOC_SCRATCH = 4 << 20
ESB_B_NK = 0
ESB_B_KN = 1
ESB_F32 = 0
ESB_BF16 = 1
ESB_F16 = 2
ESB_E4M3 = 3

_lib = None
_torch = None        # torch, once lib() has loaded (its attribute look-ups cost less than an import)


class EsbError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        msg = lib().esb_strerror(status).decode()
        if status == ESB_E_HIP:
            msg += " (hipError %d)" % lib().esb_last_hip_error()
        super().__init__("%s: %s (%d)" % (fn, msg, status))


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("N", "H", "W", "C", "K", "R", "S", "stride_h", "stride_w", "pad_h", "pad_w",
                 "groups")]


class DdaJob(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("len", ctypes.c_int64), ("n", ctypes.c_int),
                ("k_sig", ctypes.c_int), ("grid", ctypes.c_void_p), ("G", ctypes.c_int),
                ("alpha_out", ctypes.c_void_p), ("D_out", ctypes.c_void_p),
                ("grid_scale", ctypes.c_void_p)]


class ProjectJob(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("len", ctypes.c_int64), ("alpha", ctypes.c_void_p),
                ("n", ctypes.c_int), ("k_sig", ctypes.c_int), ("codes", ctypes.c_void_p)]


class PostDesc(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("relu", ctypes.c_int), ("alpha", ctypes.c_void_p), ("n", ctypes.c_int),
                ("k_sig", ctypes.c_int), ("codes", ctypes.c_void_p), ("absmax_out", ctypes.c_void_p)]


def lib():
    """Load libesb.so (after torch, so that both share one HIP runtime)."""
    global _lib, _torch
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libesb.so not built: run paper_2109_03513_amd.build.build()")
        try:
            import torch  # (loads torch's HIP runtime first)
            _torch = torch
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        f32 = ctypes.c_float
        sig = {
            "esb_version": (i32, []),
            "esb_strerror": (ctypes.c_char_p, [i32]),
            "esb_last_hip_error": (i32, []),
            "esb_valueset": (i32, [i32, i32, P, i32, P]),
            "esb_project": (i32, [P, i64, P, i32, i32, P, P]),
            "esb_dequantize": (i32, [P, i64, P, i32, i32, P, P]),
            "esb_dda_workspace_size": (sz, [i64, i32, i32, i32]),
            "esb_dda_align": (i32, [P, i64, i32, i32, P, i32, P, P, P, sz, P]),
            "esb_dda_align_noalloc": (i32, [P, i64, i32, i32, P, i32, P, P, P]),
            "esb_dda_plan_size": (sz, [i32, i32, i32]),
            "esb_dda_plan": (i32, [i32, i32, P, i32, P, sz, P]),
            "esb_dda_align_planned": (i32, [P, i64, i32, i32, P, i32, P, P, P, P, sz, P]),
            "esb_quantize_planned": (i32, [P, i64, i32, i32, P, i32, P, P, P, P, P, sz, P]),
            "esb_gemm": (i32, [i32, i32, i32, P, i64, i32, i32, P, P, i64, i32, i32, P, i32, P, P,
                               i64, P]),
            "esb_conv2d": (i32, [ctypes.POINTER(ConvDesc), P, i32, i32, P, P, i32, i32, P, P, P,
                                 P]),
            "esb_gemm_workspace_size": (sz, [i32, i32, i32, i32, i32, i32, i32]),
            "esb_gemm_ws": (i32, [i32, i32, i32, P, i64, i32, i32, P, P, i64, i32, i32, P, i32, P,
                                  P, i64, P, sz, P]),
            "esb_conv2d_workspace_size": (sz, [ctypes.POINTER(ConvDesc), i32, i32, i32, i32]),
            "esb_conv2d_ws": (i32, [ctypes.POINTER(ConvDesc), P, i32, i32, P, P, i32, i32, P, P, P,
                                    P, sz, P]),
            "esb_pack_size": (sz, [i32, i32, i32, i32]),
            "esb_pack": (i32, [P, i32, i32, i64, i32, i32, P, P]),
            "esb_gemm_packed_workspace_size": (sz, [i32, i32, i32, i32, i32, i32, i32]),
            "esb_gemm_post": (i32, [i32, i32, i32, P, i64, i32, i32, P, P, i64, i32, i32, P, i32,
                                    P, P, i64, ctypes.POINTER(PostDesc), P, sz, P]),
            "esb_conv2d_post": (i32, [ctypes.POINTER(ConvDesc), P, i32, i32, P, P, i32, i32, P, P,
                                      P, ctypes.POINTER(PostDesc), P, sz, P]),
            "esb_dda_batch_workspace_size": (sz, [i32, ctypes.POINTER(DdaJob)]),
            "esb_dda_align_batch": (i32, [i32, ctypes.POINTER(DdaJob), P, sz, P]),
            "esb_project_batch": (i32, [i32, ctypes.POINTER(ProjectJob), P]),
            "esb_maxpool2d": (i32, [P, i32, i32, i32, i32, i32, i32, i32, i32, P, P]),
            "esb_conv2d_relu_maxpool_workspace_size": (sz, [ctypes.POINTER(ConvDesc), i32, i32, i32,
                                                             i32, i32, i32, i32]),
            "esb_conv2d_relu_maxpool": (i32, [ctypes.POINTER(ConvDesc), P, i32, i32, P, P, i32, i32,
                                              P, ctypes.POINTER(PostDesc), i32, i32, i32, P, P, sz,
                                              P]),
            "esb_avgpool_global": (i32, [P, i32, i32, i32, P, P, P]),
            "esb_absmax": (i32, [P, i64, P, P]),
            "esb_dn_workspace_size": (sz, [i64]),
            "esb_dn_stats": (i32, [P, i64, P, P, sz, P]),
            "esb_project_dn": (i32, [P, i64, P, P, i32, i32, P, P]),
            "esb_dda_normal": (i32, [i32, i32, P, i32, P, P, P, P]),
            "esb_rmsnorm": (i32, [P, i64, P, i64, i32, i64, i64, P, f32, P, i64, P, i64, P, i64, P, P]),
            "esb_swiglu": (i32, [P, i64, P, i64, i32, i64, i64, P, i64, P, i64, P, P]),
            "esb_w4_size": (sz, [i32, i32, i32]),
            "esb_w4_quantize": (i32, [P, i64, i32, i32, i32, i32, P, i32, P, sz, P]),
            "esb_w4_pack": (i32, [P, i64, P, i64, i32, i32, i32, P, sz, P]),
            "esb_w4_unpack": (i32, [P, i32, i32, i32, P, i64, P, i64, P]),
            "esb_w4_gemm_workspace_size": (sz, [i32, i32, i32, i32, i32, i32]),
            "esb_w4_gemm": (i32, [i32, i32, i32, i32, P, i64, i32, P, P, P, i64, i32, P, sz, P]),
            "esb_gemm_packed": (i32, [i32, i32, i32, P, i64, i32, i32, P, P, i32, i32, P, P, P, i64,
                                      P, sz, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(fn, status):
    if status != ESB_OK:
        raise EsbError(fn, status)


def _ptr(t):
    """Address of a tensor (or None): what a c_void_p argument takes as it is."""
    return None if t is None else t.data_ptr()


def _stream(stream):
    """Handle of a stream: an int, an object with .cuda_stream, or the current one for None."""
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    torch = _torch
    if torch is None:
        import torch
    try:   # the raw handle, without building a Stream object (which costs several us a call)
        c = torch._C
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def _dev_tensor(t, dtype, name):
    torch = _torch
    if torch is None:
        import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def esb_version():
    return lib().esb_version()


def esb_valueset(n, k_sig):
    """Sorted 2^n - 1 unscaled values of Q_e (host call)."""
    out = np.zeros(256, dtype=np.float32)
    cnt = ctypes.c_int(0)
    _check("esb_valueset", lib().esb_valueset(n, k_sig, out.ctypes.data_as(ctypes.c_void_p), 256,
                                              ctypes.byref(cnt)))
    return out[:cnt.value].copy()


def esb_project(x, alpha, n, k_sig, codes=None, stream=None):
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(alpha, torch.float32, "alpha")
    if codes is None:
        codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _dev_tensor(codes, torch.uint8, "codes")
    if codes.numel() != x.numel():
        raise ValueError("codes must have as many elements as x")
    _check("esb_project", lib().esb_project(_ptr(x), x.numel(), _ptr(alpha), n, k_sig, _ptr(codes),
                                            _stream(stream)))
    return codes


def esb_dequantize(codes, alpha, n, k_sig, out=None, stream=None):
    import torch
    _dev_tensor(codes, torch.uint8, "codes")
    _dev_tensor(alpha, torch.float32, "alpha")
    if out is None:
        out = torch.empty(codes.shape, dtype=torch.float32, device=codes.device)
    _dev_tensor(out, torch.float32, "out")
    _check("esb_dequantize", lib().esb_dequantize(_ptr(codes), codes.numel(), _ptr(alpha), n, k_sig,
                                                  _ptr(out), _stream(stream)))
    return out


def esb_dda_workspace_size(length, n, k_sig, G):
    return int(lib().esb_dda_workspace_size(length, n, k_sig, G))


def esb_dda_align(x, n, k_sig, grid, alpha_out=None, D_out=None, workspace=None, stream=None,
                  want_D=True):
    """Returns (alpha_out[1] fp32 tensor, D_out[G] fp64 tensor or None)."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(grid, torch.float32, "grid")
    G = grid.numel()
    dev = x.device
    if alpha_out is None:
        alpha_out = torch.empty(1, dtype=torch.float32, device=dev)
    if D_out is None and want_D:
        D_out = torch.empty(G, dtype=torch.float64, device=dev)
    need = esb_dda_workspace_size(x.numel(), n, k_sig, G)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    _check("esb_dda_align", lib().esb_dda_align(_ptr(x), x.numel(), n, k_sig, _ptr(grid), G,
                                                _ptr(alpha_out), _ptr(D_out), _ptr(workspace),
                                                workspace.numel() * workspace.element_size(),
                                                _stream(stream)))
    return alpha_out, D_out


def esb_dda_align_noalloc(x, n, k_sig, grid, alpha_out, D_out=None, stream=None):
    """esb_dda_align with the library's static scratch (no workspace); alpha_out (and D_out,
    if given) are preallocated device tensors, so that the call allocates nothing."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(grid, torch.float32, "grid")
    _dev_tensor(alpha_out, torch.float32, "alpha_out")
    if D_out is not None:
        _dev_tensor(D_out, torch.float64, "D_out")
    _check("esb_dda_align_noalloc", lib().esb_dda_align_noalloc(
        _ptr(x), x.numel(), n, k_sig, _ptr(grid), grid.numel(), _ptr(alpha_out), _ptr(D_out),
        _stream(stream)))
    return alpha_out, D_out


def esb_dda_plan(n, k_sig, factors, plan=None, stream=None):
    """The grid-only set-up of the DDA for candidates factors[j] (device fp32), built on the
    device; returns the plan (a uint8 device tensor)."""
    import torch
    _dev_tensor(factors, torch.float32, "factors")
    G = factors.numel()
    need = int(lib().esb_dda_plan_size(n, k_sig, G))
    if need == 0:
        raise EsbError("esb_dda_plan_size", ESB_E_INVALID)
    if plan is None:
        plan = torch.empty(need, dtype=torch.uint8, device=factors.device)
    _check("esb_dda_plan", lib().esb_dda_plan(n, k_sig, _ptr(factors), G, _ptr(plan),
                                              plan.numel(), _stream(stream)))
    return plan


def esb_dda_align_planned(x, n, k_sig, plan, G, scale, alpha_out=None, D_out=None, workspace=None,
                          stream=None, want_D=True):
    """DDA over the candidates 2^E factors[j] of a plan, E the binary exponent of |scale|
    (device scalar).  Returns (alpha_out, D_out)."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(scale, torch.float32, "scale")
    dev = x.device
    if alpha_out is None:
        alpha_out = torch.empty(1, dtype=torch.float32, device=dev)
    if D_out is None and want_D:
        D_out = torch.empty(G, dtype=torch.float64, device=dev)
    if workspace is None:
        need = esb_dda_workspace_size(x.numel(), n, k_sig, G)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    _check("esb_dda_align_planned", lib().esb_dda_align_planned(
        _ptr(x), x.numel(), n, k_sig, _ptr(plan), G, _ptr(scale), _ptr(alpha_out), _ptr(D_out),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))
    return alpha_out, D_out


def esb_quantize_planned(x, n, k_sig, plan, G, scale, alpha_out=None, D_out=None, codes=None,
                         workspace=None, stream=None, want_D=True):
    """The planned DDA's alpha (and D), then the codes of x under it, in one call.
    Returns (alpha_out, D_out, codes)."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(scale, torch.float32, "scale")
    dev = x.device
    if alpha_out is None:
        alpha_out = torch.empty(1, dtype=torch.float32, device=dev)
    if D_out is None and want_D:
        D_out = torch.empty(G, dtype=torch.float64, device=dev)
    if codes is None:
        codes = torch.empty(x.shape, dtype=torch.uint8, device=dev)
    if workspace is None:
        need = esb_dda_workspace_size(x.numel(), n, k_sig, G)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    _check("esb_quantize_planned", lib().esb_quantize_planned(
        _ptr(x), x.numel(), n, k_sig, _ptr(plan), G, _ptr(scale), _ptr(alpha_out), _ptr(D_out),
        _ptr(codes), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)))
    return alpha_out, D_out, codes


def esb_gemm_workspace_size(M, N, K, nA, kA_sig, nB, kB_sig):
    return int(lib().esb_gemm_workspace_size(M, N, K, nA, kA_sig, nB, kB_sig))


def esb_conv2d_workspace_size(x_shape, w_shape, nX, kX_sig, nW, kW_sig, stride=(1, 1), pad=(0, 0),
                              groups=1):
    Nb, H, W, C = x_shape
    K, R, S, _ = w_shape
    d = ConvDesc(Nb, H, W, C, K, R, S, stride[0], stride[1], pad[0], pad[1], groups)
    return int(lib().esb_conv2d_workspace_size(ctypes.byref(d), nX, kX_sig, nW, kW_sig))


def _ws(workspace):
    """(pointer, bytes) of an optional workspace tensor."""
    if workspace is None:
        return None, 0
    return _ptr(workspace), workspace.numel() * workspace.element_size()


def esb_gemm(A, nA, kA_sig, alphaA, B, nB, kB_sig, alphaB, b_layout=ESB_B_NK, acc=None, y=None,
             want_acc=True, want_y=True, stream=None, workspace=None):
    """A: M x K codes; B: N x K (ESB_B_NK) or K x N (ESB_B_KN) codes.  Returns (acc, y).
    With a workspace tensor (esb_gemm_workspace_size bytes) the call goes to esb_gemm_ws."""
    import torch
    _dev_tensor(A, torch.uint8, "A")
    _dev_tensor(B, torch.uint8, "B")
    M, K = A.shape
    N = B.shape[0] if b_layout == ESB_B_NK else B.shape[1]
    dev = A.device
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=dev)
    if y is None and want_y:
        y = torch.empty((M, N), dtype=torch.float32, device=dev)
    lda = A.stride(0) if M else K
    ldb = B.stride(0) if B.shape[0] else 0
    if workspace is None:
        _check("esb_gemm", lib().esb_gemm(M, N, K, _ptr(A), lda, nA, kA_sig, _ptr(alphaA), _ptr(B),
                                          ldb, nB, kB_sig, _ptr(alphaB), b_layout, _ptr(acc), _ptr(y),
                                          N, _stream(stream)))
    else:
        wp, wb = _ws(workspace)
        _check("esb_gemm_ws", lib().esb_gemm_ws(M, N, K, _ptr(A), lda, nA, kA_sig, _ptr(alphaA),
                                                _ptr(B), ldb, nB, kB_sig, _ptr(alphaB), b_layout,
                                                _ptr(acc), _ptr(y), N, wp, wb, _stream(stream)))
    return acc, y


def _addr(t):
    return None if t is None else t.data_ptr()


def post_desc(alpha, n, k_sig, codes=None, a=None, b=None, residual=None, relu=False, absmax=None):
    """esb_post of device tensors: per-channel a, b, a residual in the output layout, relu, the
    output codes (uint8, output layout) under the device scalar alpha in ESB(n, k_sig), and a
    device fp32 scalar raised to max|z|."""
    return PostDesc(_addr(a), _addr(b), _addr(residual), int(bool(relu)), _addr(alpha), n, k_sig,
                    _addr(codes), _addr(absmax))


def esb_gemm_post(A, nA, kA_sig, alphaA, B, nB, kB_sig, alphaB, out_alpha, out_n, out_k_sig,
                  a=None, b=None, residual=None, relu=False, b_layout=ESB_B_NK, codes=None,
                  want_codes=True, acc=None, want_acc=False, y=None, want_y=False, workspace=None,
                  stream=None, absmax=None):
    """Contraction with the fused post-processing; returns (acc, y, codes), M x N each."""
    import torch
    _dev_tensor(A, torch.uint8, "A")
    _dev_tensor(B, torch.uint8, "B")
    M, K = A.shape
    N = B.shape[0] if b_layout == ESB_B_NK else B.shape[1]
    dev = A.device
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=dev)
    if y is None and want_y:
        y = torch.empty((M, N), dtype=torch.float32, device=dev)
    if codes is None and want_codes:
        codes = torch.empty((M, N), dtype=torch.uint8, device=dev)
    d = post_desc(out_alpha, out_n, out_k_sig, codes, a, b, residual, relu, absmax)
    lda = A.stride(0) if M else K
    ldb = B.stride(0) if B.shape[0] else 0
    wp, wb = _ws(workspace)
    _check("esb_gemm_post", lib().esb_gemm_post(M, N, K, _ptr(A), lda, nA, kA_sig, _ptr(alphaA),
                                                _ptr(B), ldb, nB, kB_sig, _ptr(alphaB), b_layout,
                                                _ptr(acc), _ptr(y), N, ctypes.byref(d), wp, wb,
                                                _stream(stream)))
    return acc, y, codes


def esb_conv2d_post(x, nX, kX_sig, alphaX, w, nW, kW_sig, alphaW, out_alpha, out_n, out_k_sig,
                    a=None, b=None, residual=None, relu=False, stride=(1, 1), pad=(0, 0),
                    groups=1, codes=None, want_codes=True, acc=None, want_acc=False, y=None,
                    want_y=False, workspace=None, stream=None, absmax=None):
    """Convolution with the fused post-processing; returns (acc, y, codes), NHWC each."""
    import torch
    _dev_tensor(x, torch.uint8, "x")
    _dev_tensor(w, torch.uint8, "w")
    Nb, H, W, C = x.shape
    K, R, S, _ = w.shape
    P, Q = conv_out_hw(H, W, R, S, stride, pad)
    dev = x.device
    if acc is None and want_acc:
        acc = torch.empty((Nb, P, Q, K), dtype=torch.int32, device=dev)
    if y is None and want_y:
        y = torch.empty((Nb, P, Q, K), dtype=torch.float32, device=dev)
    if codes is None and want_codes:
        codes = torch.empty((Nb, P, Q, K), dtype=torch.uint8, device=dev)
    pd = post_desc(out_alpha, out_n, out_k_sig, codes, a, b, residual, relu, absmax)
    d = ConvDesc(Nb, H, W, C, K, R, S, stride[0], stride[1], pad[0], pad[1], groups)
    wp, wb = _ws(workspace)
    _check("esb_conv2d_post", lib().esb_conv2d_post(ctypes.byref(d), _ptr(x), nX, kX_sig,
                                                    _ptr(alphaX), _ptr(w), nW, kW_sig,
                                                    _ptr(alphaW), _ptr(acc), _ptr(y),
                                                    ctypes.byref(pd), wp, wb, _stream(stream)))
    return acc, y, codes


def esb_conv2d_relu_maxpool(x, nX, kX_sig, alphaX, w, nW, kW_sig, alphaW, out_alpha=None,
                            out_n=5, out_k_sig=3, a=None, b=None, stride=(2, 2), pad=(3, 3),
                            pool=(3, 2, 1), y=None, want_y=True, codes=None, want_codes=False,
                            absmax=None, workspace=None, stream=None):
    """Convolution, post-processing with a ReLU and max pooling (pool = (window, stride, pad));
    returns (y, codes), each [N, PP, QQ, K] or None."""
    import torch
    _dev_tensor(x, torch.uint8, "x")
    _dev_tensor(w, torch.uint8, "w")
    Nb, H, W, C = x.shape
    K, R, S, _ = w.shape
    P, Q = conv_out_hw(H, W, R, S, stride, pad)
    PP, QQ = conv_out_hw(P, Q, pool[0], pool[0], (pool[1], pool[1]), (pool[2], pool[2]))
    dev = x.device
    if y is None and want_y:
        y = torch.empty((Nb, PP, QQ, K), dtype=torch.float32, device=dev)
    if codes is None and want_codes:
        codes = torch.empty((Nb, PP, QQ, K), dtype=torch.uint8, device=dev)
    pd = post_desc(out_alpha, out_n, out_k_sig, codes, a, b, None, True, absmax)
    d = ConvDesc(Nb, H, W, C, K, R, S, stride[0], stride[1], pad[0], pad[1], 1)
    wp, wb = _ws(workspace)
    _check("esb_conv2d_relu_maxpool", lib().esb_conv2d_relu_maxpool(
        ctypes.byref(d), _ptr(x), nX, kX_sig, _ptr(alphaX), _ptr(w), nW, kW_sig, _ptr(alphaW),
        ctypes.byref(pd), pool[0], pool[1], pool[2], _ptr(y), wp, wb, _stream(stream)))
    return y, codes


def esb_conv2d_relu_maxpool_workspace_size(x_shape, w_shape, nX, kX_sig, nW, kW_sig,
                                           stride=(2, 2), pad=(3, 3), pool=(3, 2, 1)):
    Nb, H, W, C = x_shape
    K, R, S, _ = w_shape
    d = ConvDesc(Nb, H, W, C, K, R, S, stride[0], stride[1], pad[0], pad[1], 1)
    return int(lib().esb_conv2d_relu_maxpool_workspace_size(ctypes.byref(d), nX, kX_sig, nW,
                                                             kW_sig, pool[0], pool[1], pool[2]))


def dda_jobs(specs):
    """ctypes array of esb_dda_job from (x, n, k_sig, grid, alpha_out, D_out[, grid_scale])
    tuples; with grid_scale (a device scalar) candidate j is fl32(grid_scale * grid[j])."""
    arr = (DdaJob * len(specs))()
    for i, spec in enumerate(specs):
        x, n, k_sig, grid, alpha_out, D_out = spec[:6]
        gs = spec[6] if len(spec) > 6 else None
        arr[i] = DdaJob(_addr(x), x.numel(), n, k_sig, _addr(grid), grid.numel(), _addr(alpha_out),
                        _addr(D_out), _addr(gs))
    return arr


def esb_dda_batch_workspace_size(jobs):
    return int(lib().esb_dda_batch_workspace_size(len(jobs), jobs))


def esb_dda_align_batch(jobs, workspace, stream=None):
    """DDA of every job (a dda_jobs() array) in one launch of each kernel."""
    wp, wb = _ws(workspace)
    _check("esb_dda_align_batch", lib().esb_dda_align_batch(len(jobs), jobs, wp, wb,
                                                            _stream(stream)))


def project_jobs(specs):
    """ctypes array of esb_project_job from (x, alpha, n, k_sig, codes) tuples."""
    arr = (ProjectJob * len(specs))()
    for i, (x, alpha, n, k_sig, codes) in enumerate(specs):
        arr[i] = ProjectJob(_addr(x), x.numel(), _addr(alpha), n, k_sig, _addr(codes))
    return arr


def esb_project_batch(jobs, stream=None):
    """Projection of every job (a project_jobs() array) in one launch."""
    _check("esb_project_batch", lib().esb_project_batch(len(jobs), jobs, _stream(stream)))


def esb_maxpool2d(x, window, stride, pad, out=None, stream=None):
    """NHWC fp32 max pool (padding never selected); returns out [N, P, Q, C]."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    N, H, W, C = x.shape
    P, Q = conv_out_hw(H, W, window, window, (stride, stride), (pad, pad))
    if out is None:
        out = torch.empty((N, P, Q, C), dtype=torch.float32, device=x.device)
    _dev_tensor(out, torch.float32, "out")
    _check("esb_maxpool2d", lib().esb_maxpool2d(_ptr(x), N, H, W, C, window, window, stride, pad,
                                                _ptr(out), _stream(stream)))
    return out


def esb_avgpool_global(x, out=None, absmax=None, stream=None):
    """x [N, H, W, C] (or [N, HW, C]) fp32 -> out [N, C]: fp64 sums in position order / HW."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    N, C = x.shape[0], x.shape[-1]
    HW = x.numel() // max(N * C, 1) if N * C else 1
    if out is None:
        out = torch.empty((N, C), dtype=torch.float32, device=x.device)
    _dev_tensor(out, torch.float32, "out")
    _check("esb_avgpool_global", lib().esb_avgpool_global(_ptr(x), N, HW, C, _ptr(out),
                                                          _ptr(absmax), _stream(stream)))
    return out


def esb_absmax(x, absmax, stream=None):
    """Raise the device fp32 scalar `absmax` to max |x| (the caller sets its start value)."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    _dev_tensor(absmax, torch.float32, "absmax")
    _check("esb_absmax", lib().esb_absmax(_ptr(x), x.numel(), _ptr(absmax), _stream(stream)))
    return absmax


def esb_pack_size(rows, K, n, k_sig):
    return int(lib().esb_pack_size(rows, K, n, k_sig))


def esb_pack(codes, n, k_sig, packed=None, stream=None):
    """codes: rows x K (K % 32 == 0, format inside OCP E2M1) -> rows x K/2 packed bytes."""
    import torch
    _dev_tensor(codes, torch.uint8, "codes")
    rows, K = codes.shape
    if packed is None:
        packed = torch.empty((rows, K // 2), dtype=torch.uint8, device=codes.device)
    ld = codes.stride(0) if rows else K
    _check("esb_pack", lib().esb_pack(_ptr(codes), rows, K, ld, n, k_sig, _ptr(packed),
                                      _stream(stream)))
    return packed


def esb_gemm_packed_workspace_size(M, N, K, nA, kA_sig, nB, kB_sig):
    return int(lib().esb_gemm_packed_workspace_size(M, N, K, nA, kA_sig, nB, kB_sig))


def esb_gemm_packed(A, nA, kA_sig, alphaA, B_packed, nB, kB_sig, alphaB, workspace, acc=None,
                    y=None, want_acc=True, want_y=True, stream=None):
    """A: M x K codes; B_packed: N x K/2 bytes from esb_pack.  Returns (acc, y)."""
    import torch
    _dev_tensor(A, torch.uint8, "A")
    _dev_tensor(B_packed, torch.uint8, "B_packed")
    M, K = A.shape
    N = B_packed.shape[0]
    dev = A.device
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=dev)
    if y is None and want_y:
        y = torch.empty((M, N), dtype=torch.float32, device=dev)
    lda = A.stride(0) if M else K
    wp, wb = _ws(workspace)
    _check("esb_gemm_packed", lib().esb_gemm_packed(M, N, K, _ptr(A), lda, nA, kA_sig, _ptr(alphaA),
                                                    _ptr(B_packed), nB, kB_sig, _ptr(alphaB),
                                                    _ptr(acc), _ptr(y), N, wp, wb, _stream(stream)))
    return acc, y


def esb_dn_stats(x, stats=None, workspace=None, stream=None):
    """Device fp32 [mean, std] of x (population standard deviation)."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    n = x.numel()
    if stats is None:
        stats = torch.empty(2, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(int(lib().esb_dn_workspace_size(n)), dtype=torch.uint8,
                                device=x.device)
    wp, wb = _ws(workspace)
    _check("esb_dn_stats", lib().esb_dn_stats(_ptr(x), n, _ptr(stats), wp, wb, _stream(stream)))
    return stats


def esb_project_dn(x, stats, alpha, n, k_sig, codes=None, stream=None):
    """Codes of fl32(fl32(x - mean) / fl32(std + 1e-7)) under alpha; stats = [mean, std]."""
    import torch
    _dev_tensor(x, torch.float32, "x")
    if codes is None:
        codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _check("esb_project_dn", lib().esb_project_dn(_ptr(x), x.numel(), _ptr(stats), _ptr(alpha), n,
                                                  k_sig, _ptr(codes), _stream(stream)))
    return codes


def esb_dda_normal(n, k_sig, grid, alpha_out=None, D_out=None, dD_out=None, stream=None):
    """Analytic one-sided D_j for N(0,1) over the candidates grid (device fp32); dD_out
    (optional device fp64 tensor of grid's size) receives dD/dalpha."""
    import torch
    G = grid.numel()
    if alpha_out is None:
        alpha_out = torch.empty(1, dtype=torch.float32, device=grid.device)
    if D_out is None:
        D_out = torch.empty(G, dtype=torch.float64, device=grid.device)
    _check("esb_dda_normal", lib().esb_dda_normal(n, k_sig, _ptr(grid), G, _ptr(alpha_out),
                                                  _ptr(D_out), _ptr(dD_out), _stream(stream)))
    return alpha_out, D_out


def conv_out_hw(H, W, R, S, stride, pad):
    return (H + 2 * pad[0] - R) // stride[0] + 1, (W + 2 * pad[1] - S) // stride[1] + 1


def esb_conv2d(x, nX, kX_sig, alphaX, w, nW, kW_sig, alphaW, stride=(1, 1), pad=(0, 0), groups=1,
               acc=None, y=None, want_acc=True, want_y=True, stream=None, workspace=None):
    """x: [N, H, W, C] codes (NHWC); w: [K, R, S, C/groups] codes (KRSC).  Returns (acc, y) NHWC.
    With a workspace tensor (esb_conv2d_workspace_size bytes) the call goes to esb_conv2d_ws."""
    import torch
    _dev_tensor(x, torch.uint8, "x")
    _dev_tensor(w, torch.uint8, "w")
    Nb, H, W, C = x.shape
    K, R, S, _ = w.shape
    P, Q = conv_out_hw(H, W, R, S, stride, pad)
    dev = x.device
    if acc is None and want_acc:
        acc = torch.empty((Nb, P, Q, K), dtype=torch.int32, device=dev)
    if y is None and want_y:
        y = torch.empty((Nb, P, Q, K), dtype=torch.float32, device=dev)
    d = ConvDesc(Nb, H, W, C, K, R, S, stride[0], stride[1], pad[0], pad[1], groups)
    if workspace is None:
        _check("esb_conv2d", lib().esb_conv2d(ctypes.byref(d), _ptr(x), nX, kX_sig, _ptr(alphaX),
                                              _ptr(w), nW, kW_sig, _ptr(alphaW), _ptr(acc), _ptr(y),
                                              _stream(stream)))
    else:
        wp, wb = _ws(workspace)
        _check("esb_conv2d_ws", lib().esb_conv2d_ws(ctypes.byref(d), _ptr(x), nX, kX_sig,
                                                    _ptr(alphaX), _ptr(w), nW, kW_sig, _ptr(alphaW),
                                                    _ptr(acc), _ptr(y), wp, wb, _stream(stream)))
    return acc, y


# ---- decoder operators ----------------------------------------------------------------------

_types = None        # dtype -> ESB_F32 / ESB_BF16 / ESB_F16 / ESB_E4M3


def _type(t, name, allowed):
    """Number of the tensor's (or dtype's) element type, one of `allowed`."""
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: ESB_F32, torch.bfloat16: ESB_BF16, torch.float16: ESB_F16,
                  torch.float8_e4m3fn: ESB_E4M3}
    n = _types.get(getattr(t, "dtype", t))
    if n not in allowed:
        raise TypeError("%s has an element type that this call does not take" % name)
    return n


_FLOATS = (ESB_F32, ESB_BF16, ESB_F16)


def _on(stream):
    """Context in which `stream` (an object with .cuda_stream, or a handle) is the current one: what a
    call allocates then belongs to the stream that uses it."""
    if not isinstance(stream, _torch.cuda.Stream):
        stream = _torch.cuda.ExternalStream(_stream(stream))
    return _torch.cuda.stream(stream)


def _matrix(t, name):
    """(rows, columns, pitch) of a device matrix whose columns are adjacent; rows may be apart."""
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("%s must have two dimensions" % name)
    rows, cols = shape
    sr, sc = t.stride()
    if sc != 1 and cols > 1:
        raise ValueError("%s must have adjacent columns" % name)
    if rows <= 1:
        return rows, cols, cols
    if sr < cols:
        raise ValueError("%s must not have overlapping rows" % name)
    return rows, cols, sr


def _like(t, name, rows, cols, dtype, index):
    """Pitch of a matrix that has to have this shape and type, on this device."""
    r, c, ld = _matrix(t, name)
    if r != rows or c != cols or t.dtype != dtype or t.get_device() != index:
        raise ValueError("%s must be %d x %d of %s on cuda:%d" % (name, rows, cols, dtype, index))
    return ld


def _vector(t, name, n, dtype, index):
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.get_device() != index or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous elements on cuda:%d" % (name, n, index))


def _row_outputs(x, rows, d, index, y, want_y, y8, scale, want_y8):
    """y, y8 and scale as given or new, and the pitches of y and y8."""
    ldy = ld8 = d
    if y is not None:
        ldy = _like(y, "y", rows, d, x.dtype, index)
    elif want_y:
        y = x.new_empty(rows, d)
    if y8 is not None:
        ld8 = _like(y8, "y8", rows, d, _torch.float8_e4m3fn, index)
    elif want_y8:
        y8 = x.new_empty(rows, d, dtype=_torch.float8_e4m3fn)
    if y8 is not None:
        if scale is None:
            scale = x.new_empty(rows, dtype=_torch.float32)
        else:
            _vector(scale, "scale", rows, _torch.float32, index)
    return y, ldy, y8, ld8, scale


def esb_rmsnorm(x, w, eps, residual=None, sum_out=None, want_sum=False, y=None, want_y=False,
                y8=None, scale=None, want_y8=True, stream=None):
    """Rows of z = x + residual, normalized: y = z / sqrt(mean(z^2) + eps) * w.  x, residual,
    sum_out, y: rows x d, fp32, bf16 or fp16 (row pitches allowed); w: d fp32, or None.
    Returns (sum, y, y8, scale): z and y in x's type, and y as float8_e4m3fn under one fp32 scale
    per row; what is neither given nor wanted is None."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_rmsnorm(x, w, eps, residual, sum_out, want_sum, y, want_y, y8, scale, want_y8)
    rows, d, ldx = _matrix(x, "x")
    t = _type(x, "x", _FLOATS)
    index = x.get_device()
    ldr = lds = 0
    if residual is not None:
        ldr = _like(residual, "residual", rows, d, x.dtype, index)
    if w is not None:
        _vector(w, "w", d, _torch.float32, index)
    if sum_out is not None:
        lds = _like(sum_out, "sum_out", rows, d, x.dtype, index)
    elif want_sum:
        sum_out, lds = x.new_empty(rows, d), d
    y, ldy, y8, ld8, scale = _row_outputs(x, rows, d, index, y, want_y, y8, scale, want_y8)
    st = L.esb_rmsnorm(x.data_ptr(), ldx, _addr(residual), ldr, t, rows, d, _addr(w), eps,
                       _addr(sum_out), lds, _addr(y), ldy, _addr(y8), ld8, _addr(scale),
                       _stream(None))
    if st:
        raise EsbError("esb_rmsnorm", st)
    return sum_out, y, y8, scale


def esb_swiglu(gate, up, y=None, want_y=False, y8=None, scale=None, want_y8=True, stream=None):
    """gate / (1 + exp(-gate)) * up, rows x d; returns (y, y8, scale) as esb_rmsnorm does."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_swiglu(gate, up, y, want_y, y8, scale, want_y8)
    rows, d, ldg = _matrix(gate, "gate")
    t = _type(gate, "gate", _FLOATS)
    index = gate.get_device()
    ldu = _like(up, "up", rows, d, gate.dtype, index)
    y, ldy, y8, ld8, scale = _row_outputs(gate, rows, d, index, y, want_y, y8, scale, want_y8)
    st = L.esb_swiglu(gate.data_ptr(), ldg, up.data_ptr(), ldu, t, rows, d, _addr(y), ldy, _addr(y8),
                      ld8, _addr(scale), _stream(None))
    if st:
        raise EsbError("esb_swiglu", st)
    return y, y8, scale


def esb_w4_size(N, K, group):
    return int(lib().esb_w4_size(N, K, group))


def _w4_buffer(w4, N, K, group, like):
    need = esb_w4_size(N, K, group)
    if w4 is None:
        if need == 0 and N and K:
            raise EsbError("esb_w4_size", ESB_E_INVALID)
        return like.new_empty(max(need, 1), dtype=_torch.uint8)
    return _w4_check(w4, like.get_device())


def _w4_check(w4, index):
    if not isinstance(w4, _torch.Tensor) or not w4.is_cuda:
        raise TypeError("w4 must be a CUDA (HIP) tensor")
    if w4.dtype != _torch.uint8 or w4.get_device() != index or not w4.is_contiguous():
        raise ValueError("w4 must be contiguous uint8 on cuda:%d" % index)
    return w4


def _w4_holds(L, w4, N, K, group):
    need = L.esb_w4_size(N, K, group)
    if w4.numel() < need or (need == 0 and N and K):
        raise EsbError("esb_w4_size", ESB_E_WORKSPACE if need else ESB_E_INVALID)


def esb_w4_quantize(w, group, factors=None, w4=None, stream=None):
    """4-bit codes and group scales of w (N x K, fp32, bf16 or fp16), packed: a uint8 tensor of
    esb_w4_size(N, K, group) bytes.  factors: device fp32 candidates of the scale, as multiples
    of max|w| / 6 of the group (None: 1)."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_w4_quantize(w, group, factors, w4)
    N, K, ld = _matrix(w, "w")
    t = _type(w, "w", _FLOATS)
    if factors is not None:
        _vector(factors, "factors", factors.numel(), _torch.float32, w.get_device())
    w4 = _w4_buffer(w4, N, K, group, w)
    st = L.esb_w4_quantize(w.data_ptr(), ld, t, N, K, group, _addr(factors),
                           1 if factors is None else factors.numel(), w4.data_ptr(), w4.numel(),
                           _stream(None))
    if st:
        raise EsbError("esb_w4_quantize", st)
    return w4


def esb_w4_pack(codes, alpha, group, w4=None, stream=None):
    """The packed form of ESB(4,1) codes (N x K uint8) and bf16 scales (N x ceil(K / group))."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_w4_pack(codes, alpha, group, w4)
    N, K, ldc = _matrix(codes, "codes")
    if codes.dtype != _torch.uint8:
        raise TypeError("codes must be uint8")
    lda = _like(alpha, "alpha", N, -(-K // group) if group > 0 else 0, _torch.bfloat16,
                codes.get_device())
    w4 = _w4_buffer(w4, N, K, group, codes)
    st = L.esb_w4_pack(codes.data_ptr(), ldc, alpha.data_ptr(), lda, N, K, group, w4.data_ptr(),
                       w4.numel(), _stream(None))
    if st:
        raise EsbError("esb_w4_pack", st)
    return w4


def esb_w4_unpack(w4, N, K, group, values=None, alpha=None, stream=None):
    """(values, alpha): the unscaled values (N x K float8_e4m3fn, exact) and the group scales
    (N x ceil(K / group) bf16) of packed weights."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_w4_unpack(w4, N, K, group, values, alpha)
    index = w4.get_device() if isinstance(w4, _torch.Tensor) else -1
    _w4_check(w4, index)
    _w4_holds(L, w4, N, K, group)
    groups = -(-K // group) if group > 0 else 0
    ldv, lda = K, groups
    if values is None:
        values = w4.new_empty(N, K, dtype=_torch.float8_e4m3fn)
    else:
        ldv = _like(values, "values", N, K, _torch.float8_e4m3fn, index)
    if alpha is None:
        alpha = w4.new_empty(N, groups, dtype=_torch.bfloat16)
    else:
        lda = _like(alpha, "alpha", N, groups, _torch.bfloat16, index)
    st = L.esb_w4_unpack(w4.data_ptr(), N, K, group, values.data_ptr(), ldv, alpha.data_ptr(), lda,
                         _stream(None))
    if st:
        raise EsbError("esb_w4_unpack", st)
    return values, alpha


def esb_w4_gemm_workspace_size(M, N, K, group, x_type, y_type):
    return int(lib().esb_w4_gemm_workspace_size(M, N, K, group, x_type, y_type))


def esb_w4_gemm(x, w4, N, group, x_scale=None, y_dtype=None, y=None, workspace=None, stream=None):
    """y = x W^T for x (M x K: bf16, fp16, or float8_e4m3fn with x_scale, M fp32) and packed
    weights W (N x K); y in y_dtype (None: x's type; bf16 for float8).  workspace: at least
    esb_w4_gemm_workspace_size() bytes; without one the call allocates what it needs from torch."""
    L = _lib or lib()
    if stream is not None:
        with _on(stream):
            return esb_w4_gemm(x, w4, N, group, x_scale, y_dtype, y, workspace)
    M, K, ldx = _matrix(x, "x")
    tx = _type(x, "x", (ESB_F32, ESB_BF16, ESB_F16, ESB_E4M3))   # fp32: the library's refusal
    index = x.get_device()
    _w4_check(w4, index)
    _w4_holds(L, w4, N, K, group)
    if x_scale is not None:
        _vector(x_scale, "x_scale", M, _torch.float32, index)
    ldy = N
    if y is None:
        if y_dtype is None:
            y_dtype = _torch.bfloat16 if tx == ESB_E4M3 else x.dtype
        ty = _type(y_dtype, "y", _FLOATS)
        y = x.new_empty(M, N, dtype=y_dtype)
    else:
        ty = _type(y, "y", _FLOATS)
        ldy = _like(y, "y", M, N, y_dtype or y.dtype, index)
    if workspace is None:
        need = L.esb_w4_gemm_workspace_size(M, N, K, group, tx, ty)
        if need:
            workspace = x.new_empty(need, dtype=_torch.uint8)
    else:
        if not isinstance(workspace, _torch.Tensor) or not workspace.is_cuda:
            raise TypeError("workspace must be a CUDA (HIP) tensor")
        if workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous on cuda:%d" % index)
    wp, wb = _ws(workspace)
    st = L.esb_w4_gemm(M, N, K, group, x.data_ptr(), ldx, tx, _addr(x_scale), w4.data_ptr(),
                       y.data_ptr(), ldy, ty, wp, wb, _stream(None))
    if st:
        raise EsbError("esb_w4_gemm", st)
    return y
