"""Thin binding over libwcc.so (the C ABI of include/wcc.h): argument marshalling only.

Every step runs in the library's CUDA kernels; torch is used for device memory and the current stream.
There is no fallback: if the library is missing, or a call returns an error code, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwcc.so")

F32, BF16 = 0, 1
_STATUS = {0: "ok", 1: "null pointer", 2: "bad shape", 3: "k out of range", 4: "bad bits", 5: "bad dtype",
           6: "misaligned pointer", 7: "workspace too small", 8: "CUDA error", 9: "device wait timed out",
           10: "non-finite input", 11: "adapter index out of range"}
MAX_RANK = 64

EXPORTS = ("wcc_staged_workspace_bytes", "wcc_forward_staged", "wcc_workspace_bytes", "wcc_select_workspace_bytes", "wcc_haar_fwd", "wcc_haar_inv", "wcc_select_topk",
           "wcc_forward", "wcc_forward_debug", "wcc_kpad", "wcc_last_status", "wcc_status_str",
           "wcc_profile_enable", "wcc_profile_read", "wcc_kernel_launches", "wcc_select_topk_static",
           "wcc_debug_set_wait_limit", "wcc_debug_wait_selftest", "wcc_debug_select", "wcc_forward_ex", "wcc_chain_workspace_bytes",
           "wcc_chain_forward", "wcc_select_bitmap_workspace_bytes", "wcc_select_topk_bitmap",
           "wcc_padded_workspace_bytes", "wcc_forward_padded", "wcc_dwconv_haar_fwd", "wcc_block_workspace_bytes",
           "wcc_block_forward", "wcc_dwt_fwd", "wcc_dwt_inv", "wcc_wavelet_workspace_bytes", "wcc_forward_wavelet",
           "wcc_layernorm_fwd", "wcc_layernorm_bwd_workspace_bytes", "wcc_layernorm_bwd", "wcc_adapters_workspace_bytes",
           "wcc_adapters_fwd", "wcc_adapters_bwd", "wcc_forward_check", "wcc_debug_adapters_path", "wcc_debug_layernorm_path")
STATIC_SCRATCH_BYTES = 512 * 1024
STAGES = ("haar_fwd_norms", "select_topk", "weight_quant", "gather_quant", "contract", "scatter_inv")   # wcc_forward_staged
FUSED_STAGES = ("clear", "haar_norms", "select_topk", "fused_pass2")                                      # wcc_forward


class WccError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__("%s: %s (status %d)" % (where, _STATUS.get(code, "?"), code))
        self.code = code


class Taps(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("coef", "nrm2", "idx", "Xq", "Xb", "scale_a", "Wq", "scale_w", "acc")]


class Options(C.Structure):
    _fields_ = [("alpha", C.c_float), ("weight_bits", C.c_int), ("relu", C.c_int), ("residual", C.c_void_p),
                ("Wq", C.c_void_p), ("scale_w", C.c_void_p)]


class ChainLayer(C.Structure):
    _fields_ = [("Wt", C.c_void_p), ("Cin", C.c_int), ("Cout", C.c_int), ("alpha", C.c_float), ("relu", C.c_int)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (``python -m paper_2205_12268_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError("libwcc.so is not built: run `python -m paper_2205_12268_b200.build` "
                                    "(needs nvcc; there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        i, vp, sz = C.c_int, C.c_void_p, C.c_size_t
        L.wcc_workspace_bytes.restype = sz
        L.wcc_workspace_bytes.argtypes = [i] * 9
        L.wcc_staged_workspace_bytes.restype = sz
        L.wcc_staged_workspace_bytes.argtypes = [i] * 9
        L.wcc_select_workspace_bytes.restype = sz
        L.wcc_select_workspace_bytes.argtypes = [i, i]
        L.wcc_kpad.restype = i
        L.wcc_kpad.argtypes = [i, i]
        L.wcc_haar_fwd.restype = i
        L.wcc_haar_fwd.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp]
        L.wcc_haar_inv.restype = i
        L.wcc_haar_inv.argtypes = [vp, i, i, i, i, i, i, vp, vp]
        L.wcc_select_topk.restype = i
        L.wcc_select_topk.argtypes = [vp, i, i, i, vp, vp, vp, sz, vp]
        L.wcc_select_topk_static.restype = i
        L.wcc_select_topk_static.argtypes = [vp, i, i, i, vp, vp, vp]
        fwd = [vp, vp, i, i, i, i, i, i, i, i, vp, i, vp, sz, vp]
        L.wcc_forward.restype = i
        L.wcc_forward.argtypes = fwd
        L.wcc_forward_debug.restype = i
        L.wcc_forward_debug.argtypes = fwd + [C.POINTER(Taps)]
        L.wcc_forward_staged.restype = i
        L.wcc_forward_staged.argtypes = fwd + [C.POINTER(Taps)]
        L.wcc_forward_ex.restype = i
        L.wcc_forward_ex.argtypes = fwd + [C.POINTER(Options), C.POINTER(Taps)]
        L.wcc_select_bitmap_workspace_bytes.restype = sz
        L.wcc_select_bitmap_workspace_bytes.argtypes = [i, i, i]
        L.wcc_select_topk_bitmap.restype = i
        L.wcc_select_topk_bitmap.argtypes = [vp, i, i, i, vp, vp, vp, sz, vp]
        L.wcc_padded_workspace_bytes.restype = sz
        L.wcc_padded_workspace_bytes.argtypes = [i] * 9
        L.wcc_forward_padded.restype = i
        L.wcc_forward_padded.argtypes = fwd
        L.wcc_dwconv_haar_fwd.restype = i
        L.wcc_dwconv_haar_fwd.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp]
        L.wcc_block_workspace_bytes.restype = sz
        L.wcc_block_workspace_bytes.argtypes = [i] * 9
        L.wcc_block_forward.restype = i
        L.wcc_block_forward.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp, i, vp, sz, vp]
        fp = C.POINTER(C.c_float)
        L.wcc_dwt_fwd.restype = i
        L.wcc_dwt_fwd.argtypes = [vp, i, i, i, i, i, i, fp, fp, i, vp, vp, vp, sz, vp]
        L.wcc_dwt_inv.restype = i
        L.wcc_dwt_inv.argtypes = [vp, i, i, i, i, i, i, fp, fp, i, vp, vp, sz, vp]
        L.wcc_wavelet_workspace_bytes.restype = sz
        L.wcc_wavelet_workspace_bytes.argtypes = [i] * 9
        L.wcc_forward_wavelet.restype = i
        L.wcc_forward_wavelet.argtypes = [vp, vp, i, i, i, i, i, i, i, i, fp, fp, fp, fp, i, vp, i, vp, sz, vp, C.POINTER(Taps)]
        L.wcc_chain_workspace_bytes.restype = sz
        L.wcc_chain_workspace_bytes.argtypes = [C.POINTER(ChainLayer), i, i, i, i, i, i, i, i]
        L.wcc_chain_forward.restype = i
        L.wcc_chain_forward.argtypes = [vp, C.POINTER(ChainLayer), i, i, i, i, i, i, i, vp, i, vp, sz, vp]
        _operator_prototypes(L)
        L.wcc_profile_enable.restype = i
        L.wcc_profile_enable.argtypes = [i]
        L.wcc_profile_read.restype = i
        L.wcc_profile_read.argtypes = [C.POINTER(C.c_float)]
        L.wcc_kernel_launches.restype = C.c_ulonglong
        L.wcc_kernel_launches.argtypes = []
        L.wcc_debug_set_wait_limit.restype = i
        L.wcc_debug_set_wait_limit.argtypes = [C.c_uint]
        L.wcc_debug_wait_selftest.restype = i
        L.wcc_debug_wait_selftest.argtypes = [vp]
        L.wcc_debug_select.restype = i
        L.wcc_debug_select.argtypes = [vp, i, i, vp, vp, i, i, vp, vp, vp, vp]
        L.wcc_status_str.restype = C.c_char_p
        L.wcc_status_str.argtypes = [i]
        _lib = L
    return _lib


def _operator_prototypes(L):
    """Layer norm, adapters and the status word."""
    i, vp, sz, f = C.c_int, C.c_void_p, C.c_size_t, C.c_float
    L.wcc_layernorm_fwd.restype = i
    L.wcc_layernorm_fwd.argtypes = [vp, vp, vp, i, i, i, i, f, i, vp, vp, vp, vp]
    L.wcc_layernorm_bwd_workspace_bytes.restype = sz
    L.wcc_layernorm_bwd_workspace_bytes.argtypes = [i] * 5
    L.wcc_layernorm_bwd.restype = i
    L.wcc_layernorm_bwd.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp, vp, sz, vp]
    L.wcc_adapters_workspace_bytes.restype = sz
    L.wcc_adapters_workspace_bytes.argtypes = [i] * 9
    L.wcc_adapters_fwd.restype = i
    L.wcc_adapters_fwd.argtypes = [vp] * 6 + [i] * 8 + [vp, vp, sz, vp]
    L.wcc_adapters_bwd.restype = i
    L.wcc_adapters_bwd.argtypes = [vp] * 7 + [i] * 8 + [vp, vp, vp, vp, sz, vp]
    L.wcc_forward_check.restype = i
    L.wcc_forward_check.argtypes = [vp, vp] + [i] * 8 + [vp, i, vp, sz, C.POINTER(Options), C.POINTER(Taps)]
    L.wcc_debug_adapters_path.restype = i
    L.wcc_debug_adapters_path.argtypes = [i] * 8 + [vp, i]
    L.wcc_debug_layernorm_path.restype = i
    L.wcc_debug_layernorm_path.argtypes = [i] * 6
    L.wcc_last_status.restype = i
    L.wcc_last_status.argtypes = [vp]


def _check(code: int, where: str):
    if code != 0:
        raise WccError(code, where)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("activations must be float32 or bfloat16, got %s" % t.dtype)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """Handle of the current stream, where torch has a call for it without the Stream object of current_stream()."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, name: str):
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError("%s must be a contiguous CUDA tensor" % name)


def _room(t: torch.Tensor, n: int, like: torch.Tensor, name: str):
    """t holds at least n elements of `like`'s type, one after the other on `like`'s device: the kernels go by the sizes of the call, not by t's."""
    if not (t.is_cuda and t.is_contiguous() and t.dtype == like.dtype and t.device == like.device and t.numel() >= n):
        raise ValueError("%s must be contiguous, of at least %d elements of %s on %s" % (name, n, like.dtype, like.device))


def workspace_bytes(N, Cin, Cout, H, W, levels, k, bits, dt) -> int:
    return int(lib().wcc_workspace_bytes(N, Cin, Cout, H, W, levels, k, bits, dt))


def kpad(Cin: int, bits: int) -> int:
    return int(lib().wcc_kpad(Cin, bits))


def haar_fwd(x: torch.Tensor, levels: int, want_norms: bool = True):
    """x [N][C][H][W] -> (coef fp32 [N][C][H][W] quadrant layout, nrm2 fp32 [N][H*W] or None)."""
    _dev(x, "x")
    N, Cc, H, W = x.shape
    coef = torch.empty((N, Cc, H, W), dtype=torch.float32, device=x.device)
    nrm2 = torch.empty((N, H * W), dtype=torch.float32, device=x.device) if want_norms else None
    _check(lib().wcc_haar_fwd(x.data_ptr(), N, Cc, H, W, levels, _dt(x), coef.data_ptr(), _ptr(nrm2), _stream()),
           "wcc_haar_fwd")
    return coef, nrm2


def dwconv_haar_fwd(u: torch.Tensor, Wdw: torch.Tensor, levels: int):
    """Depthwise 3x3 convolution (Wdw fp32 [C][3][3]) fused with the forward transform -> (coef, nrm2) as ``haar_fwd``."""
    _dev(u, "u")
    _dev(Wdw, "Wdw")
    N, Cc, H, W = u.shape
    if Wdw.dtype != torch.float32 or tuple(Wdw.shape) != (Cc, 3, 3):
        raise ValueError("Wdw must be float32 [C][3][3]")
    coef = torch.empty((N, Cc, H, W), dtype=torch.float32, device=u.device)
    nrm2 = torch.empty((N, H * W), dtype=torch.float32, device=u.device)
    _check(lib().wcc_dwconv_haar_fwd(u.data_ptr(), Wdw.data_ptr(), N, Cc, H, W, levels, _dt(u), coef.data_ptr(),
                                     nrm2.data_ptr(), _stream()), "wcc_dwconv_haar_fwd")
    return coef, nrm2


def _taps(f):
    import numpy as np
    a = np.ascontiguousarray(f, dtype=np.float32)
    return a, a.ctypes.data_as(C.POINTER(C.c_float))


def dwt_fwd(x: torch.Tensor, levels: int, dec_lo, dec_hi):
    """Generic wavelet transform (host filter arrays, see wcc.h) -> (coef fp32, nrm2 fp32 [N][P])."""
    _dev(x, "x")
    N, Cc, H, W = x.shape
    lo, plo = _taps(dec_lo)
    hi, phi = _taps(dec_hi)
    coef = torch.empty((N, Cc, H, W), dtype=torch.float32, device=x.device)
    nrm2 = torch.empty((N, H * W), dtype=torch.float32, device=x.device)
    ws = torch.empty((N * Cc * H * W * 4,), dtype=torch.uint8, device=x.device)
    _check(lib().wcc_dwt_fwd(x.data_ptr(), N, Cc, H, W, levels, _dt(x), plo, phi, lo.size, coef.data_ptr(), nrm2.data_ptr(),
                             ws.data_ptr(), ws.numel(), _stream()), "wcc_dwt_fwd")
    return coef, nrm2


def dwt_inv(coef: torch.Tensor, levels: int, rec_lo, rec_hi, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    _dev(coef, "coef")
    N, Cc, H, W = coef.shape
    lo, plo = _taps(rec_lo)
    hi, phi = _taps(rec_hi)
    out = torch.empty((N, Cc, H, W), dtype=dtype, device=coef.device)
    ws = torch.empty((2 * (N * Cc * H * W * 4 + 256),), dtype=torch.uint8, device=coef.device)
    _check(lib().wcc_dwt_inv(coef.data_ptr(), N, Cc, H, W, levels, _dt(out), plo, phi, lo.size, out.data_ptr(),
                             ws.data_ptr(), ws.numel(), _stream()), "wcc_dwt_inv")
    return out


def forward_wavelet(x: torch.Tensor, Wt: torch.Tensor, levels: int, k: int, bits: int, bank, taps: bool = False):
    """The layer with another wavelet: ``bank`` = (dec_lo, dec_hi, rec_lo, rec_hi) host arrays of equal even length."""
    _dev(x, "x")
    _dev(Wt, "Wt")
    N, Cin, H, W = x.shape
    Cout = Wt.shape[0]
    f = [_taps(b) for b in bank]
    nbytes = int(lib().wcc_wavelet_workspace_bytes(N, Cin, Cout, H, W, levels, k, bits, _dt(x)))
    if nbytes == 0:
        raise WccError(2, "wcc_wavelet_workspace_bytes")
    ws = torch.empty((nbytes,), dtype=torch.uint8, device=x.device)
    y = torch.empty((N, Cout, H, W), dtype=x.dtype, device=x.device)
    t, s = {}, None
    if taps:
        P, M, kp = H * W, N * k, kpad(Cin, bits)
        t = dict(coef=torch.empty((N, Cin, P), dtype=torch.float32, device=x.device),
                 nrm2=torch.empty((N, P), dtype=torch.float32, device=x.device),
                 idx=torch.empty((N, k), dtype=torch.int32, device=x.device),
                 acc=torch.empty((M, Cout), dtype=torch.int32, device=x.device))
        if bits >= 2:
            t["Xq"] = torch.empty((M, kp), dtype=torch.int8, device=x.device)
        s = Taps(**{name: _ptr(t.get(name)) for name, _ in Taps._fields_})
    _check(lib().wcc_forward_wavelet(x.data_ptr(), Wt.data_ptr(), N, Cin, Cout, H, W, levels, k, bits, f[0][1], f[1][1], f[2][1],
                                     f[3][1], f[0][0].size, y.data_ptr(), _dt(x), ws.data_ptr(), nbytes, _stream(),
                                     C.byref(s) if s is not None else None), "wcc_forward_wavelet")
    return (y, t) if taps else y


class Block:
    """The inverted residual block y = x + WCC(W3, dw3x3(Wdw, WCC(W1, x))) (wcc_block_forward); the workspace, which
    also holds the expanded map, is allocated once, here."""

    def __init__(self, x: torch.Tensor, W1: torch.Tensor, Wdw: torch.Tensor, W3: torch.Tensor, levels: int, k: int, bits: int = 8):
        _dev(x, "x")
        for t, name in ((W1, "W1"), (Wdw, "Wdw"), (W3, "W3")):
            _dev(t, name)
            if t.dtype != torch.float32:
                raise TypeError("%s must be float32" % name)
        self.N, self.C, self.H, self.W = x.shape
        self.E = W1.shape[0]
        if tuple(W1.shape) != (self.E, self.C) or tuple(Wdw.shape) != (self.E, 3, 3) or tuple(W3.shape) != (self.C, self.E):
            raise ValueError("W1 [E][C], Wdw [E][3][3], W3 [C][E] expected")
        self.W1, self.Wdw, self.W3, self.levels, self.k, self.bits, self.dt = W1, Wdw, W3, levels, k, bits, _dt(x)
        n = int(lib().wcc_block_workspace_bytes(self.N, self.C, self.E, self.H, self.W, levels, k, bits, self.dt))
        if n == 0:
            raise WccError(2, "wcc_block_workspace_bytes")
        self.ws = Workspace(n, x.device)

    def __call__(self, x: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
        _dev(x, "x")
        if _dt(x) != self.dt:
            raise ValueError("x must have the type the block was made for")
        n = self.N * self.C * self.H * self.W
        _room(x, n, x, "x")
        if y is None:
            y = torch.empty_like(x)
        else:
            _room(y, n, x, "y")
        _check(lib().wcc_block_forward(x.data_ptr(), self.W1.data_ptr(), self.Wdw.data_ptr(), self.W3.data_ptr(), self.N,
                                       self.C, self.E, self.H, self.W, self.levels, self.k, self.bits, y.data_ptr(), self.dt,
                                       self.ws.buf.data_ptr(), self.ws.nbytes, _stream()), "wcc_block_forward")
        return y


def haar_inv(coef: torch.Tensor, levels: int, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    _dev(coef, "coef")
    if coef.dtype != torch.float32:
        raise TypeError("coef must be float32")
    N, Cc, H, W = coef.shape
    out = torch.empty((N, Cc, H, W), dtype=dtype, device=coef.device)
    _check(lib().wcc_haar_inv(coef.data_ptr(), N, Cc, H, W, levels, _dt(out), out.data_ptr(), _stream()), "wcc_haar_inv")
    return out


def select_topk(nrm2: torch.Tensor, k: int):
    """nrm2 fp32 [N][P] -> (idx int32 [N][k] ascending, tau fp32 [N])."""
    _dev(nrm2, "nrm2")
    if nrm2.dtype != torch.float32:
        raise TypeError("nrm2 must be float32")
    N, P = nrm2.shape
    idx = torch.empty((N, max(k, 1)), dtype=torch.int32, device=nrm2.device)
    tau = torch.empty((N,), dtype=torch.float32, device=nrm2.device)
    nbytes = int(lib().wcc_select_workspace_bytes(N, P))
    ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=nrm2.device)
    _check(lib().wcc_select_topk(nrm2.data_ptr(), N, P, k, idx.data_ptr(), tau.data_ptr(), ws.data_ptr(), nbytes, _stream()),
           "wcc_select_topk")
    return idx, tau


def select_topk_bitmap(nrm2: torch.Tensor, k: int):
    """nrm2 fp32 [N][P] -> (bitmap int32 [N][ceil(P/32)] with bit p % 32 of word p // 32 set for kept p, tau fp32 [N])."""
    _dev(nrm2, "nrm2")
    N, P = nrm2.shape
    bitmap = torch.empty((N, (P + 31) // 32), dtype=torch.int32, device=nrm2.device)
    tau = torch.empty((N,), dtype=torch.float32, device=nrm2.device)
    nbytes = int(lib().wcc_select_bitmap_workspace_bytes(N, P, k))
    ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=nrm2.device)
    _check(lib().wcc_select_topk_bitmap(nrm2.data_ptr(), N, P, k, bitmap.data_ptr(), tau.data_ptr(), ws.data_ptr(), nbytes,
                                        _stream()), "wcc_select_topk_bitmap")
    return bitmap, tau


def forward_padded(x: torch.Tensor, Wt: torch.Tensor, levels: int, k: int, bits: int = 8) -> torch.Tensor:
    """The layer on a map whose sides need not be multiples of 2^levels (zero padding, see wcc_forward_padded);
    k counts positions of the padded map."""
    _dev(x, "x")
    _dev(Wt, "Wt")
    N, Cin, H, W = x.shape
    Cout = Wt.shape[0]
    nbytes = int(lib().wcc_padded_workspace_bytes(N, Cin, Cout, H, W, levels, k, bits, _dt(x)))
    if nbytes == 0:
        raise WccError(2, "wcc_padded_workspace_bytes")
    ws = torch.empty((nbytes,), dtype=torch.uint8, device=x.device)
    y = torch.empty((N, Cout, H, W), dtype=x.dtype, device=x.device)
    _check(lib().wcc_forward_padded(x.data_ptr(), Wt.data_ptr(), N, Cin, Cout, H, W, levels, k, bits, y.data_ptr(), _dt(x),
                                    ws.data_ptr(), nbytes, _stream()), "wcc_forward_padded")
    return y


def select_topk_static(nrm2: torch.Tensor, k: int, idx: torch.Tensor, tau: torch.Tensor):
    """``select_topk`` for callers that cannot provide scratch memory: the library's built-in scratch array is used
    and nothing is allocated, here or in the library (the caller passes the output tensors).  Raises ``WccError``
    with code 7 when N and P need more than ``STATIC_SCRATCH_BYTES``.  Calls on one device share the scratch, so
    they must not overlap on the GPU."""
    _dev(nrm2, "nrm2")
    N, P = nrm2.shape
    _check(lib().wcc_select_topk_static(nrm2.data_ptr(), N, P, k, idx.data_ptr(), tau.data_ptr(), _stream()),
           "wcc_select_topk_static")
    return idx, tau


class Workspace:
    """Caller-owned scratch for ``forward``; reuse it across calls of the same (or smaller) problem."""

    def __init__(self, nbytes: int, device):
        self.nbytes = int(nbytes)
        self.buf = torch.empty((max(self.nbytes, 256),), dtype=torch.uint8, device=device)

    @classmethod
    def for_problem(cls, x: torch.Tensor, Cout: int, levels: int, k: int, bits: int, staged: bool = False):
        N, Cin, H, W = x.shape
        fn = lib().wcc_staged_workspace_bytes if staged else lib().wcc_workspace_bytes
        n = int(fn(N, Cin, Cout, H, W, levels, k, bits, _dt(x)))
        if n == 0:
            raise WccError(2, "wcc_workspace_bytes")
        return cls(n, x.device)

    @classmethod
    def for_layernorm_backward(cls, x: torch.Tensor):
        n = int(lib().wcc_layernorm_bwd_workspace_bytes(*_map_shape(x, "x"), _dt(x)))
        if n == 0:
            raise WccError(2, "wcc_layernorm_bwd_workspace_bytes")
        return cls(n, x.device)


def _map_shape(x: torch.Tensor, name: str):
    """(N, C, H, W) of a map [N][C][H][W] or of rows [N][C], which are maps of one position."""
    _dev(x, name)
    if x.dim() == 4:
        return x.shape
    if x.dim() != 2:
        raise ValueError("%s must be [N][C][H][W] or [N][C]" % name)
    return (x.shape[0], x.shape[1], 1, 1)


def _here(x: torch.Tensor) -> int:
    """The device of a call's map.  The library launches on the current device's current stream: maps of another device are refused."""
    dev = x.get_device()
    if dev != torch.cuda.current_device():
        raise ValueError("the map is on cuda:%d, which is not the current device" % dev)
    return dev


def _same(t: torch.Tensor, like: torch.Tensor, dev: int, name: str, what: str) -> int:
    """The address of t, which must have `like`'s shape and type on device `dev`, contiguous as every map."""
    if not (t.get_device() == dev and t.is_contiguous() and t.dtype == like.dtype and t.shape == like.shape):
        raise ValueError("%s must be contiguous, of the shape, type and device of %s" % (name, what))
    return t.data_ptr()


def _floats(t, n: int, dev: int, name: str, rows: int = 0):
    """The address of t, None or fp32 [n] (with `rows`: [rows][n]) on device `dev`."""
    if t is None:
        return None
    if not (t.get_device() == dev and t.is_contiguous() and t.dtype == torch.float32 and t.shape == ((rows, n) if rows else (n,))):
        raise ValueError("%s must be contiguous float32 %s on the device of the map" % (name, [rows, n] if rows else [n]))
    return t.data_ptr()


def layernorm(x: torch.Tensor, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None, eps: float = 1e-5,
              y: torch.Tensor | None = None, stats: bool = False):
    """Layer norm over the channels of a map [N][C][H][W] (or of rows [N][C]), fp32 ``gamma`` and ``beta`` [C] or None.
    Returns y (``y`` may be x), or with ``stats`` (y, mean, rstd), the statistics fp32 [N][H*W] as the backward pass reads them."""
    N, Cc, H, W = _map_shape(x, "x")
    dt, dev = _dt(x), _here(x)
    pg, pb = _floats(gamma, Cc, dev, "gamma"), _floats(beta, Cc, dev, "beta")
    if y is None:
        y = torch.empty_like(x)
        py = y.data_ptr()
    else:
        py = _same(y, x, dev, "y", "x")
    mean = rstd = pm = pr = None
    if stats:
        mean, rstd = x.new_empty((N, H * W), dtype=torch.float32), x.new_empty((N, H * W), dtype=torch.float32)
        pm, pr = mean.data_ptr(), rstd.data_ptr()
    _check(lib().wcc_layernorm_fwd(x.data_ptr(), pg, pb, N, Cc, H, W, eps, dt, py, pm, pr, _stream()), "wcc_layernorm_fwd")
    return (y, mean, rstd) if stats else y


def layernorm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, gamma: torch.Tensor | None = None,
                       dx: torch.Tensor | None = None, params: bool = True, ws: Workspace | None = None):
    """The gradients of ``layernorm``: (dx, dgamma, dbeta), the last two fp32 [C] and None without ``params``.
    ``dx`` may be dy or x.  ``ws`` is a ``Workspace.for_layernorm_backward``, allocated here if it is not given."""
    N, Cc, H, W = _map_shape(x, "x")
    dt, dev = _dt(x), _here(x)
    pdy, pg = _same(dy, x, dev, "dy", "x"), _floats(gamma, Cc, dev, "gamma")
    pm, pr = _floats(mean, H * W, dev, "mean", N), _floats(rstd, H * W, dev, "rstd", N)
    if dx is None:
        dx = torch.empty_like(x)
        pdx = dx.data_ptr()
    else:
        pdx = _same(dx, x, dev, "dx", "x")
    dgamma = dbeta = pdg = pdb = pw = None
    nw = 0
    if params:
        dgamma, dbeta = x.new_empty((Cc,), dtype=torch.float32), x.new_empty((Cc,), dtype=torch.float32)
        if ws is None:
            ws = Workspace.for_layernorm_backward(x)
        pdg, pdb, pw, nw = dgamma.data_ptr(), dbeta.data_ptr(), ws.buf.data_ptr(), ws.nbytes
    _check(lib().wcc_layernorm_bwd(pdy, x.data_ptr(), pg, pm, pr, N, Cc, H, W, dt, pdx, pdg, pdb, pw, nw, _stream()), "wcc_layernorm_bwd")
    return dx, dgamma, dbeta


class Adapters:
    """Low-rank adapters beside a shared projection: factors ``A`` [R][rank][Cin] and ``B`` [R][Cout][rank] of the maps' type, ``scale`` fp32 [R]
    or None for 1.  The tensors are kept, not copied: a call sees what they hold when it runs.

    ``adapters(x, ids)`` -> base + scale * B (A x) with the adapter ids[n] (int32 [N] on the device, negative: none) for image n of x
    [N][Cin][H][W] (or of rows [N][Cin]); ``adapters.backward(dy, x, ids)`` -> (dx, dA, dB).  See wcc_adapters_fwd and wcc_adapters_bwd."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None):
        for t, name in ((A, "A"), (B, "B")):
            _dev(t, name)
            if t.dim() != 3:
                raise ValueError("A [R][rank][Cin] and B [R][Cout][rank] expected")
        self.dt = _dt(A)
        self.R, self.rank, self.Cin = A.shape
        self.Cout = B.shape[1]
        if B.dtype != A.dtype or B.device != A.device or tuple(B.shape) != (self.R, self.Cout, self.rank):
            raise ValueError("B must be [R][Cout][rank] of A's type on A's device")
        if not 1 <= self.rank <= MAX_RANK:
            raise ValueError("the rank must be 1 to %d" % MAX_RANK)
        _floats(scale, self.R, A.get_device(), "scale")
        self.A, self.B, self.scale = A, B, scale
        self._ws_bytes = {}

    def workspace(self, x: torch.Tensor, backward: bool = True) -> Workspace:
        """Scratch for calls on maps of x's shape; that for the backward pass also serves the forward pass."""
        N, _, H, W = self._shape(x)
        n = self._bytes(N, H, W, False)
        return Workspace(max(n, self._bytes(N, H, W, True)) if backward else n, x.device)

    def _bytes(self, N, H, W, backward):
        n = self._ws_bytes.get((N, H, W, backward))
        if n is None:
            n = int(lib().wcc_adapters_workspace_bytes(N, self.Cin, self.Cout, H, W, self.R, self.rank, self.dt, int(backward)))
            if n == 0:
                raise WccError(2, "wcc_adapters_workspace_bytes")
            self._ws_bytes[N, H, W, backward] = n
        return n

    def _scratch(self, x, N, H, W, backward, ws):
        if ws is not None:
            return ws.buf, ws.nbytes
        n = self._bytes(N, H, W, backward)
        return x.new_empty((n,), dtype=torch.uint8), n

    def _shape(self, x):
        shape = _map_shape(x, "x")
        if x.dtype != self.A.dtype or shape[1] != self.Cin or x.get_device() != self.A.get_device():
            raise ValueError("x must have the adapters' type, Cin channels and device")
        return shape

    @staticmethod
    def _ids(ids, N, dev):
        if not (ids.get_device() == dev and ids.is_contiguous() and ids.dtype == torch.int32 and ids.shape == (N,)):
            raise ValueError("ids must be contiguous int32 [N] on the device of the map")
        return ids.data_ptr()

    @staticmethod
    def _map(t, x, C, dev, name):
        """The address of a map of x's sizes with C channels; None stays None."""
        if t is None:
            return None
        if not (t.get_device() == dev and t.is_contiguous() and t.dtype == x.dtype and t.dim() == x.dim() and t.shape[0] == x.shape[0] and
                t.shape[1] == C and t.shape[2:] == x.shape[2:]):
            raise ValueError("%s must be a contiguous map of %d channels with x's sizes, type and device" % (name, C))
        return t.data_ptr()

    def __call__(self, x: torch.Tensor, ids: torch.Tensor, base: torch.Tensor | None = None, y: torch.Tensor | None = None,
                 ws: Workspace | None = None) -> torch.Tensor:
        N, _, H, W = self._shape(x)
        dev, px = _here(x), x.data_ptr()
        pi, pb = self._ids(ids, N, dev), self._map(base, x, self.Cout, dev, "base")
        if y is None:
            y = x.new_empty((N, self.Cout) + tuple(x.shape[2:]))
        py = self._map(y, x, self.Cout, dev, "y")
        if py == px:
            raise ValueError("y must not be x")
        buf, n = self._scratch(x, N, H, W, False, ws)
        _check(lib().wcc_adapters_fwd(px, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scale), pi, pb, N, self.Cin, self.Cout, H, W, self.R,
                                      self.rank, self.dt, py, buf.data_ptr(), n, _stream()), "wcc_adapters_fwd")
        return y

    def backward(self, dy: torch.Tensor, x: torch.Tensor, ids: torch.Tensor, base: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                 params: bool = True, ws: Workspace | None = None):
        """(dx, dA, dB): dx = base + the adapters' part of the map's gradient, dA and dB fp32 in the factors' shapes (None without ``params``)."""
        N, _, H, W = self._shape(x)
        dev, px = _here(x), x.data_ptr()
        pi, pdy, pb = self._ids(ids, N, dev), self._map(dy, x, self.Cout, dev, "dy"), self._map(base, x, self.Cin, dev, "base")
        if dx is None:
            dx = torch.empty_like(x)
        pdx = self._map(dx, x, self.Cin, dev, "dx")
        if pdx == px or pdx == pdy:
            raise ValueError("dx must not be x or dy")
        dA = x.new_empty(self.A.shape, dtype=torch.float32) if params else None
        dB = x.new_empty(self.B.shape, dtype=torch.float32) if params else None
        buf, n = self._scratch(x, N, H, W, True, ws)
        _check(lib().wcc_adapters_bwd(pdy, px, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scale), pi, pb, N, self.Cin, self.Cout, H, W, self.R,
                                      self.rank, self.dt, pdx, _ptr(dA), _ptr(dB), buf.data_ptr(), n, _stream()), "wcc_adapters_bwd")
        return dx, dA, dB


def forward(x: torch.Tensor, Wt: torch.Tensor | None, levels: int, k: int, bits: int = 8, y: torch.Tensor | None = None,
            ws: Workspace | None = None, taps: bool = False, staged: bool = False, alpha: float = 0.0, wbits: int = 0,
            relu: bool = False, residual: torch.Tensor | None = None, Wq: torch.Tensor | None = None,
            scale_w: torch.Tensor | None = None, adapters: Adapters | None = None, ids: torch.Tensor | None = None):
    """The WCC layer.  Returns y, or (y, dict of intermediate tensors) when ``taps`` is set (True: all of them; or an
    iterable of names out of coef, nrm2, idx, acc, Xq / Xb, scale_a, Wq, scale_w).
    ``staged`` selects wcc_forward_staged (every intermediate in memory) instead of the fused wcc_forward.
    ``alpha``, ``wbits``, ``relu``, ``residual``, ``Wq`` + ``scale_w``: the options of wcc_forward_ex (see wcc.h);
    with pre-quantized weights ``Wt`` may be None.
    ``adapters`` with ``ids`` (int32 [N], negative: none): low-rank adapters beside the layer's projection.  Their sum (and ``residual``) is written to y
    in the map's type and enters the layer as its residual, so the ReLU comes after it.  They run in ``ws`` where it is large enough, else in scratch of
    their own.  A call that is refused leaves y as it is.  Without ``adapters``, ``ids`` are not read."""
    _dev(x, "x")
    N, Cin, H, W = x.shape
    if adapters is not None:
        if ids is None:
            raise ValueError("adapters need ids")
        if staged:
            raise ValueError("options are only available on the fused path")
    use_ex = bool(alpha > 0.0 or wbits or relu or residual is not None or Wq is not None or adapters is not None)
    if Wq is not None:
        _dev(Wq, "Wq")
        if scale_w is not None:
            _dev(scale_w, "scale_w")
        Cout = Wq.shape[0]
    else:
        _dev(Wt, "Wt")
        if Wt.dtype != torch.float32:
            raise TypeError("Wt must be float32")
        Cout = Wt.shape[0]
        if Wt.shape[1] != Cin:
            raise ValueError("Wt must be [Cout][Cin]")
    if adapters is not None and (adapters.Cin != Cin or adapters.Cout != Cout):
        raise ValueError("the adapters must have the layer's channels")
    if use_ex and staged:
        raise ValueError("options are only available on the fused path")
    if residual is not None:
        _dev(residual, "residual")
        if residual.shape != (N, Cout, H, W) or residual.dtype != x.dtype:
            raise ValueError("residual must have the output's shape and type")
    if y is None:
        y = torch.empty((N, Cout, H, W), dtype=x.dtype, device=x.device)
    else:
        _room(y, N * Cout * H * W, x, "y")
    if ws is None:
        ws = Workspace.for_problem(x, Cout, levels, k, bits, staged=staged)
    args = (x.data_ptr(), _ptr(Wt), N, Cin, Cout, H, W, levels, k, bits, y.data_ptr(), _dt(x),
            ws.buf.data_ptr(), ws.nbytes, _stream())
    opt = Options(float(alpha), int(wbits), int(bool(relu)), _ptr(residual), _ptr(Wq), _ptr(scale_w)) if use_ex else None
    t, s = _tap_tensors(x, Cout, k, bits, taps) if taps else (None, None)
    if adapters is not None:
        # the layer's residual is what the adapters leave in y: their launch comes after all that could refuse the layer
        opt.residual = y.data_ptr()
        _check(lib().wcc_forward_check(*args[:-1], C.byref(opt), C.byref(s) if taps else None), "wcc_forward_check")
        adapters(x, ids, base=residual, y=y, ws=ws if ws.nbytes >= adapters._bytes(N, H, W, False) else None)
    if not taps:
        if staged:
            _check(lib().wcc_forward_staged(*args, None), "wcc_forward_staged")
        elif use_ex:
            _check(lib().wcc_forward_ex(*args, C.byref(opt), None), "wcc_forward_ex")
        else:
            _check(lib().wcc_forward(*args), "wcc_forward")
        return y
    if staged:
        _check(lib().wcc_forward_staged(*args, C.byref(s)), "wcc_forward_staged")
    elif use_ex:
        _check(lib().wcc_forward_ex(*args, C.byref(opt), C.byref(s)), "wcc_forward_ex")
    else:
        _check(lib().wcc_forward_debug(*args, C.byref(s)), "wcc_forward_debug")
    return y, t


def _tap_tensors(x: torch.Tensor, Cout: int, k: int, bits: int, taps):
    """Tensors for the intermediates of a layer that ``taps`` names (True: all), and the Taps that point at them."""
    N, Cin, H, W = x.shape
    P, M, kp = H * W, N * k, kpad(Cin, bits)
    dev = x.device
    t = dict(coef=torch.empty((N, Cin, P), dtype=torch.float32, device=dev),
             nrm2=torch.empty((N, P), dtype=torch.float32, device=dev),
             idx=torch.empty((N, k), dtype=torch.int32, device=dev),
             acc=torch.empty((M, Cout), dtype=torch.int32, device=dev))
    if bits >= 2:
        t.update(Xq=torch.empty((M, kp), dtype=torch.int8, device=dev), scale_a=torch.empty((1,), dtype=torch.float32, device=dev),
                 Wq=torch.empty((Cout, kp), dtype=torch.int8, device=dev), scale_w=torch.empty((Cout,), dtype=torch.float32, device=dev))
    else:
        t.update(Xb=torch.empty((M, kp), dtype=torch.bfloat16, device=dev))
    if taps is not True:
        t = {name: v for name, v in t.items() if name in set(taps)}
    for name in ("Xq", "Xb", "acc"):          # every row is a kept position and gets written; start from zeros anyway
        if name in t:
            t[name].zero_()
    return t, Taps(**{name: _ptr(t.get(name)) for name, _ in Taps._fields_})


class Chain:
    """A chain of pointwise WCC layers (wcc_chain_forward): ``weights[i]`` is layer i's fp32 [Cout][Cin] device tensor;
    a ReLU follows every layer but (unless ``relu_last``) the last; ``alphas[i]`` > 0 fixes layer i's clipping parameter.
    The workspace (intermediate maps included) is allocated once, here.

    ``norms[i]`` = (gamma, beta, eps): layer i's input is normalised over its channels first (``layernorm``; gamma and beta may be None);
    ``adapters[i]``: ``Adapters`` beside layer i, taken by the ``ids`` of the call (not read where no layer has any).  Either list may hold None for layers
    without.  Such a chain runs layer by layer."""

    def __init__(self, x: torch.Tensor, weights, levels: int, k: int, bits: int = 8, relu_last: bool = False, alphas=None, norms=None,
                 adapters=None):
        _dev(x, "x")
        self.N, cin, self.H, self.W = x.shape
        self.levels, self.k, self.bits, self.dt = levels, k, bits, _dt(x)
        self.weights = list(weights)
        n = len(self.weights)
        self.layers = (ChainLayer * n)()
        for i, Wt in enumerate(self.weights):
            _dev(Wt, "weights[%d]" % i)
            if Wt.dtype != torch.float32 or Wt.shape[1] != cin:
                raise ValueError("weights[%d] must be float32 [Cout][%d]" % (i, cin))
            self.layers[i] = ChainLayer(Wt.data_ptr(), cin, Wt.shape[0], 0.0 if alphas is None else float(alphas[i]),
                                        int(relu_last or i + 1 < n))
            cin = Wt.shape[0]
        self.Cout = cin
        nbytes = int(lib().wcc_chain_workspace_bytes(self.layers, n, self.N, self.H, self.W, levels, k, bits, self.dt))
        if nbytes == 0:
            raise WccError(2, "wcc_chain_workspace_bytes")
        self.norms, self.adapters = ([None] * n if v is None else list(v) for v in (norms, adapters))
        if len(self.norms) != n or len(self.adapters) != n:
            raise ValueError("norms and adapters must have an entry for each layer")
        self.plain = not any(v is not None for v in self.norms + self.adapters)
        if not self.plain:
            self._prepare(x)
            return
        self.ws = Workspace(nbytes, x.device)

    def _prepare(self, x: torch.Tensor):
        """What a chain that runs layer by layer keeps: two intermediate maps, a normalised one, and scratch for any of its calls."""
        n, wide, normed, nbytes = len(self.weights), 0, 0, 0
        for i, layer in enumerate(self.layers):
            Cin, Cout = layer.Cin, layer.Cout
            if i + 1 < n:
                wide = max(wide, Cout)
            if self.norms[i] is not None:
                gamma, beta, _ = self.norms[i]
                _floats(gamma, Cin, x.get_device(), "norms[%d]: gamma" % i)
                _floats(beta, Cin, x.get_device(), "norms[%d]: beta" % i)
                normed = max(normed, Cin)
            if self.adapters[i] is not None:
                a = self.adapters[i]
                if (a.Cin, a.Cout, a.dt) != (Cin, Cout, self.dt) or a.A.device != x.device:
                    raise ValueError("adapters[%d] must have the layer's channels and the map's type and device" % i)
                nbytes = max(nbytes, a._bytes(self.N, self.H, self.W, False))
            nbytes = max(nbytes, int(lib().wcc_workspace_bytes(self.N, Cin, Cout, self.H, self.W, self.levels, self.k, self.bits, self.dt)))
        self.ws = Workspace(nbytes, x.device)
        room = self.N * self.H * self.W
        self.between = [x.new_empty((room * wide,)) for _ in range(2 if n > 2 else 1)] if n > 1 else []
        self.normed = x.new_empty((room * normed,)) if normed else None

    def _run(self, x: torch.Tensor, y: torch.Tensor, ids) -> torch.Tensor:
        n = len(self.weights)
        if ids is None and any(a is not None for a in self.adapters):
            raise ValueError("adapters need ids")
        for i, layer in enumerate(self.layers):
            shape = (self.N, layer.Cin, self.H, self.W)
            if self.norms[i] is not None:
                gamma, beta, eps = self.norms[i]
                x = layernorm(x, gamma, beta, eps, y=self.normed[:x.numel()].view(shape))
            out = y if i + 1 == n else self.between[i % len(self.between)][:self.N * layer.Cout * self.H * self.W].view(self.N, layer.Cout, self.H, self.W)
            x = forward(x, self.weights[i], self.levels, self.k, self.bits, y=out, ws=self.ws, alpha=layer.alpha, relu=bool(layer.relu),
                        adapters=self.adapters[i], ids=ids)
        return x

    def __call__(self, x: torch.Tensor, y: torch.Tensor | None = None, ids: torch.Tensor | None = None) -> torch.Tensor:
        _dev(x, "x")
        if _dt(x) != self.dt or (not self.plain and tuple(x.shape) != (self.N, self.layers[0].Cin, self.H, self.W)):
            raise ValueError("x must have the shape and type the chain was made for")
        _room(x, self.N * self.layers[0].Cin * self.H * self.W, x, "x")
        if y is None:
            y = torch.empty((self.N, self.Cout, self.H, self.W), dtype=x.dtype, device=x.device)
        else:
            _room(y, self.N * self.Cout * self.H * self.W, x, "y")
        if not self.plain:
            return self._run(x, y, ids)
        _check(lib().wcc_chain_forward(x.data_ptr(), self.layers, len(self.weights), self.N, self.H, self.W, self.levels,
                                       self.k, self.bits, y.data_ptr(), self.dt, self.ws.buf.data_ptr(), self.ws.nbytes,
                                       _stream()), "wcc_chain_forward")
        return y


def last_status() -> int:
    """Synchronises the current stream and returns (and clears) the device status word."""
    return int(lib().wcc_last_status(_stream()))


def debug_set_wait_limit(polls: int):
    """Polls every device-side wait makes before it gives up (0 restores the default)."""
    _check(lib().wcc_debug_set_wait_limit(int(polls)), "wcc_debug_set_wait_limit")


def debug_wait_selftest():
    """Enqueues one warp that waits on a barrier nobody arrives on (it gives up after the wait limit)."""
    _check(lib().wcc_debug_wait_selftest(_stream()), "wcc_debug_wait_selftest")


def debug_select(nrm2, k: int, hist11, hist16, want_rank: bool, thr, rank, idx, late: bool = False):
    """The selection inside a layer on one image's norms and the caller's histograms of them (wcc_debug_select)."""
    _check(lib().wcc_debug_select(nrm2.data_ptr(), nrm2.numel(), k, hist11.data_ptr(), hist16.data_ptr(), int(want_rank), int(late), thr.data_ptr(),
                                  rank.data_ptr(), idx.data_ptr(), _stream()), "wcc_debug_select")


def profile_enable(on: bool):
    _check(lib().wcc_profile_enable(int(on)), "wcc_profile_enable")


def profile_read():
    """Milliseconds of each stage (see ``STAGES``) of the last ``forward`` issued with profiling on."""
    ms = (C.c_float * len(STAGES))()
    _check(lib().wcc_profile_read(ms), "wcc_profile_read")
    return [float(v) for v in ms]


def kernel_launches() -> int:
    return int(lib().wcc_kernel_launches())
