"""Binding of libbnn's C ABI (include/bnn.h), by ctypes and, for short calls, a native module: argument marshalling only.

Tensors are ``torch`` CUDA (ROCm) tensors used purely as device buffers; every function enqueues
on torch's current stream of the tensor's device and returns the output tensor(s).  Shapes and
dtypes are checked here, everything else by the library, whose status codes are raised as
``BnnError``.
"""
from __future__ import annotations

import collections
import contextlib
import ctypes
import importlib
import math
import os
import sys
import warnings

import torch

__all__ = ["BnnError", "lib_path", "load", "PAD_MINUS_ONE", "PAD_EXCLUDE", "PATH_AUTO", "PATH_VALU", "PATH_MFMA",
           "nwords", "round_up", "bmm", "bmm_thr", "bconv", "bconv_thr", "threshold_pack", "pack_u8", "pack_f32",
           "unpack_i32", "tile_b", "bmm_tiled", "bmm_thr_tiled", "panels_from_rows", "rows_from_panels", "bmm_panels", "bmm_thr_panels", "probe_load_stride", "probe_pipeline", "probe_pipeline_enqueue", "PROBES", "sign_pack_f32", "bmm_general_f32", "bconv_general_f32", "maxpool_or", "conv_f32_thr", "conv_f32_split_thr", "bwn_conv_thr", "head_f32", "Net", "Cache4", "rotary", "rotary_frequencies", "token_logprobs", "TokenLogprobs", "EXPORTS", "bmm_kernel_name", "bconv_kernel_name"]

PAD_MINUS_ONE, PAD_EXCLUDE = 0, 1
PATH_AUTO, PATH_VALU, PATH_MFMA = 0, 1, 2

_HERE = os.path.dirname(os.path.abspath(__file__))

# every symbol include/bnn.h declares
EXPORTS = ["bnn_status_string", "bnn_version", "bnn_bmm_kernel_name", "bnn_bconv_kernel_name", "bnn_bmm_kernel_name_out", "bnn_bconv_kernel_name_out", "bnn_bconv_kernel_name_ex", "bnn_bmm", "bnn_bmm_ex", "bnn_bmm_thr", "bnn_bmm_thr_ex",
           "bnn_bconv", "bnn_bconv_ex", "bnn_bconv_thr", "bnn_bconv_thr_ex", "bnn_threshold_pack", "bnn_pack_u8",
           "bnn_pack_f32", "bnn_tile_b", "bnn_bmm_tiled", "bnn_bmm_thr_tiled", "bnn_panels_from_rows", "bnn_rows_from_panels", "bnn_bmm_panels", "bnn_bmm_thr_panels", "bnn_probe_load_stride", "bnn_probe_pipeline", "bnn_sign_pack_f32", "bnn_bmm_general_workspace_bytes", "bnn_bmm_general_f32",
           "bnn_bconv_general_workspace_bytes", "bnn_bconv_general_f32", "bnn_unpack_i32", "bnn_maxpool_or", "bnn_conv_f32_thr", "bnn_conv_f32_split_workspace_bytes", "bnn_conv_f32_split_thr", "bnn_conv_f32_split_thr_ex", "bnn_bwn_workspace_bytes", "bnn_bwn_conv_thr", "bnn_head_f32", "bnn_net_create",
           "bnn_net_destroy", "bnn_net_input_u8", "bnn_net_input_bits", "bnn_net_input_conv_f32", "bnn_net_input_bwn_f32", "bnn_net_add_fc",
           "bnn_net_add_conv", "bnn_net_add_pool", "bnn_net_add_block", "bnn_net_add_head_f32", "bnn_net_workspace_bytes",
           "bnn_net_forward", "bnn_net_forward_static", "bnn_static_workspace_init", "bnn_net_forward_persistent", "bnn_net_persistent_status", "bnn_net_fc_run", "bnn_net_layer_bits",
           "bnn_rotary", "bnn_cache4_record_bytes", "bnn_cache4_write", "bnn_cache4_write_rotary", "bnn_cache4_read", "bnn_cache4_select_workspace_bytes", "bnn_cache4_select",
           "bnn_cache4_attend_workspace_bytes", "bnn_cache4_attend", "bnn_cache4_weigh_workspace_bytes", "bnn_cache4_weigh", "bnn_cache4_heaviest_workspace_bytes", "bnn_cache4_heaviest", "bnn_cache4_move",
           "bnn_token_logprobs_workspace_bytes", "bnn_token_logprobs"]


class BnnError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (what, _status_string(status), status))


def lib_path() -> str:
    return os.path.join(_HERE, "libbnn.so")


_lib = None


def load() -> ctypes.CDLL:
    """Loads libbnn.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError("libbnn.so is not built: run `python -m paper_2006_16578_amd.build` "
                              "(or __graft_entry__.build()) first")
        lib = ctypes.CDLL(path)
        lib.bnn_status_string.restype = ctypes.c_char_p
        lib.bnn_status_string.argtypes = [ctypes.c_int]
        lib.bnn_bmm_kernel_name.restype = ctypes.c_char_p
        lib.bnn_bconv_kernel_name.restype = ctypes.c_char_p
        lib.bnn_bmm_kernel_name_out.restype = ctypes.c_char_p
        lib.bnn_bconv_kernel_name_out.restype = ctypes.c_char_p
        lib.bnn_bconv_kernel_name_ex.restype = ctypes.c_char_p
        lib.bnn_bwn_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_conv_f32_split_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_bmm_general_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_bconv_general_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_cache4_record_bytes.restype = ctypes.c_size_t
        lib.bnn_cache4_select_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_cache4_attend_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_cache4_heaviest_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_cache4_weigh_workspace_bytes.restype = ctypes.c_size_t
        lib.bnn_token_logprobs_workspace_bytes.restype = ctypes.c_size_t
        for name in EXPORTS:
            getattr(lib, name)          # fail loudly on a missing export
        _lib = lib
    return _lib


# The native module behind the calls whose kernels are short (csrc/bnn_python.cpp): each function there does what its namesake here does with
# its defaults, in a third of the host time, or returns None for whatever is out of the ordinary, and the code here goes on.
# bmm_thr of 8 x 4096 x 4096, passes queued one after another: 7.4 -> 4.0 to 4.8 us (which, differs from process to process).
_native = None


class _PythonOnly:
    """In the native module's place where it does not load: every call goes on in Python."""

    def __getattr__(self, name):
        return lambda *args: None


def _native_stamp() -> str:
    """What a build of the native module is good for: the torch and the interpreter it was compiled against."""
    return "torch %s, Python %d.%d" % (torch.__version__, sys.version_info[0], sys.version_info[1])


def _native_module():
    """The native module, initialised; raises ImportError if it is not built, or built for another torch or interpreter."""
    module = importlib.import_module("._native", __package__)
    if module.built_for != _native_stamp():
        raise ImportError("_native.so was built for %s, this is %s" % (module.built_for, _native_stamp()))
    lib = load()
    stream = _raw_stream if _raw_stream is not None else lambda index: torch.cuda.current_stream(index).cuda_stream
    module.init({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS}, stream, _check)
    return module


def _load_native():
    """Sets _native: the module, or what makes every call go by ctypes if that does not load (said once)."""
    global _native
    load()
    try:
        _native = _native_module()
    except ImportError as e:
        warnings.warn("short calls take about 3 us longer: %s (run `python -m paper_2006_16578_amd.build`)" % e, RuntimeWarning, stacklevel=3)
        _native = _PythonOnly()
    return _native


def _status_string(status: int) -> str:
    try:
        return load().bnn_status_string(status).decode()
    except Exception:  # pragma: no cover
        return "?"


def _check(status: int, what: str) -> None:
    if status != 0:
        raise BnnError(status, what)


def bmm_kernel_name(M: int, N: int, K: int, path: int = PATH_AUTO, int32_out: bool = False, program: bool = False) -> str:
    """program: the name also tells which of the kernels with this wave tile it is (BNN_NAME_PROGRAM)."""
    return load().bnn_bmm_kernel_name_out(int(M), int(N), int(K), int(path), int(bool(int32_out)) | 2 * int(bool(program))).decode()


def bconv_kernel_name(N, H, W, C, O, k, stride, pad, path: int = PATH_AUTO, int32_out: bool = False,
                      pad_mode: int = PAD_MINUS_ONE, shortcut: bool = False, pool2: bool = False, residual: bool = False,
                      keep_sum: bool = False, residual32: bool = False) -> str:
    """Of a convolution in a layer chain -- shortcut: a residual block's that also adds a 1x1 shortcut; residual / keep_sum: one that
    adds the running 16-bit sum / keeps its own; pool2: a 2x2 pooling layer follows (the name ends in "_pool2" if the
    convolution's kernel stores the pooled bits).  residual32: bconv_thr with an int32 residual ("_stream": a kernel for streamed
    residuals)."""
    return load().bnn_bconv_kernel_name_ex(int(N), int(H), int(W), int(C), int(O), int(k), int(stride), int(pad), int(pad_mode),
                                           int(path), int(bool(int32_out)), int(bool(shortcut)) | 2 * int(bool(pool2)) | 4 * int(bool(residual))
                                           | 8 * int(bool(keep_sum)) | 16 * int(bool(residual32))).decode()


def nwords(nbits: int) -> int:
    return (int(nbits) + 31) // 32


def round_up(v: int, m: int) -> int:
    return (int(v) + m - 1) // m * m


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


# What a call costs on the host counts: a small product runs 4 us on the GPU.  The two helpers below ask torch for the current
# device and the raw stream only (0.3 us; a device context manager and a Stream object per call took 3.1 of 10 us).
# (a private function of torch: without it the Stream object serves)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor):
    """The current stream of t's device."""
    if _raw_stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)
    return ctypes.c_void_p(_raw_stream(t.get_device()))


_STAY = contextlib.nullcontext()


def _on(t: torch.Tensor):
    """Context in which t's device is the current one."""
    return _STAY if torch.cuda.current_device() == t.get_device() else torch.cuda.device(t.device)


def _dev(t: torch.Tensor, dtype, ndim=None, name="tensor"):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a device tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if ndim is not None and t.dim() != ndim:
        raise ValueError("%s must have %d dimensions" % (name, ndim))
    return t


_BITS = torch.int32   # packed words travel as int32 tensors (torch has no uint32 arithmetic; only the bytes matter)


def bmm(A, B, K: int, out=None, path: int = PATH_AUTO):
    """C[i][j] = sum_k a[i][k] b[j][k]; A [M][lda_w], B [N][ldb_w] packed int32 words -> int32 [M][N]."""
    if out is None:
        done = (_native or _load_native()).bmm(A, B, K, path)
        if done is not None:
            return done
    _dev(A, _BITS, 2, "A"); _dev(B, _BITS, 2, "B")
    M, lda = A.shape
    N, ldb = B.shape
    C = torch.empty((M, N), dtype=torch.int32, device=A.device) if out is None else _dev(out, torch.int32, 2, "out")
    with _on(A):
        _check(load().bnn_bmm_ex(_ptr(A), _ptr(B), _ptr(C), M, N, int(K), lda, ldb, C.shape[1], int(path), _stream(A)), "bnn_bmm")
    return C


def bmm_thr(A, B, thr, K: int, ldcb_w: int | None = None, out=None, path: int = PATH_AUTO):
    """Fused BMM + threshold: bits [M][ldcb_w], bit j = (C[i][j] >= thr[j])."""
    if out is None and ldcb_w is None:
        done = (_native or _load_native()).bmm_thr(A, B, thr, K, path)
        if done is not None:
            return done
    _dev(A, _BITS, 2, "A"); _dev(B, _BITS, 2, "B"); _dev(thr, torch.int32, 1, "thr")
    M, lda = A.shape
    N, ldb = B.shape
    if thr.shape[0] != N:
        raise ValueError("thr must have N entries")
    ldcb_w = round_up(nwords(N), 4) if ldcb_w is None else int(ldcb_w)
    Cb = torch.empty((M, ldcb_w), dtype=_BITS, device=A.device) if out is None else _dev(out, _BITS, 2, "out")
    with _on(A):
        _check(load().bnn_bmm_thr_ex(_ptr(A), _ptr(B), _ptr(thr), _ptr(Cb), M, N, int(K), lda, ldb, Cb.shape[1], int(path),
                                     _stream(A)), "bnn_bmm_thr")
    return Cb


def _conv_dims(x, filt, C, stride, pad):
    _dev(x, _BITS, 4, "x"); _dev(filt, _BITS, 4, "filt")
    N, H, W, cw = x.shape
    O, k, k2, cwf = filt.shape
    if k != k2 or cw != cwf or cw != nwords(C):
        raise ValueError("x [N][H][W][cw], filt [O][k][k][cw] with cw = ceil(C/32) expected")
    if stride < 1:                       # the library rejects it; keep the shapes computable
        return N, H, W, O, k, 1, 1
    P = (H + 2 * pad - k) // stride + 1
    Q = (W + 2 * pad - k) // stride + 1
    return N, H, W, O, k, P, Q


def bconv(x, filt, C: int, stride: int, pad: int, pad_mode: int = PAD_MINUS_ONE, out=None, path: int = PATH_AUTO):
    """int32 [N][P][Q][O] = cross-correlation of packed x [N][H][W][cw] with filt [O][k][k][cw]."""
    if out is None:
        done = (_native or _load_native()).bconv(x, filt, C, stride, pad, pad_mode, path)
        if done is not None:
            return done
    N, H, W, O, k, P, Q = _conv_dims(x, filt, C, stride, pad)
    y = torch.empty((N, max(P, 0), max(Q, 0), O), dtype=torch.int32, device=x.device) if out is None else out
    with _on(x):
        _check(load().bnn_bconv_ex(_ptr(x), _ptr(filt), _ptr(y), N, H, W, int(C), O, k, int(stride), int(pad),
                                   int(pad_mode), int(path), _stream(x)), "bnn_bconv")
    return y


def bconv_thr(x, filt, thr, C: int, stride: int, pad: int, pad_mode: int = PAD_MINUS_ONE, residual=None,
              want_sum: bool = False, sum_out=None, out=None, path: int = PATH_AUTO):
    """Fused conv (+ int32 residual) + threshold -> bits [N][P][Q][ow]; optionally also the int32 sum."""
    if out is None and sum_out is None:
        done = (_native or _load_native()).bconv_thr(x, filt, thr, C, stride, pad, pad_mode, residual, want_sum, path)
        if done is not None:
            return done
    N, H, W, O, k, P, Q = _conv_dims(x, filt, C, stride, pad)
    _dev(thr, torch.int32, 1, "thr")
    if residual is not None:
        _dev(residual, torch.int32, 4, "residual")
        if tuple(residual.shape) != (N, P, Q, O):
            raise ValueError("residual must be [N][P][Q][O]")
    if want_sum and sum_out is None:
        sum_out = torch.empty((N, P, Q, O), dtype=torch.int32, device=x.device)
    bits = torch.empty((N, max(P, 0), max(Q, 0), nwords(O)), dtype=_BITS, device=x.device) if out is None else out
    with _on(x):
        _check(load().bnn_bconv_thr_ex(_ptr(x), _ptr(filt), _ptr(residual), _ptr(sum_out), _ptr(thr), _ptr(bits), N, H, W,
                                       int(C), O, k, int(stride), int(pad), int(pad_mode), int(path), _stream(x)),
               "bnn_bconv_thr")
    return (bits, sum_out) if sum_out is not None else bits


def threshold_pack(X, thr, ldb_w: int | None = None):
    if ldb_w is None:
        done = (_native or _load_native()).threshold_pack(X, thr)
        if done is not None:
            return done
    _dev(X, torch.int32, None, "X"); _dev(thr, torch.int32, 1, "thr")
    cols = X.shape[-1]
    rows = X.numel() // cols
    ldb_w = nwords(cols) if ldb_w is None else int(ldb_w)
    bits = torch.empty(tuple(X.shape[:-1]) + (ldb_w,), dtype=_BITS, device=X.device)
    with _on(X):
        _check(load().bnn_threshold_pack(_ptr(X), _ptr(thr), _ptr(bits), ctypes.c_int64(rows), cols, cols, ldb_w, _stream(X)),
               "bnn_threshold_pack")
    return bits


def pack_u8(x, thr: int, ldb_w: int | None = None):
    _dev(x, torch.uint8, 2, "x")
    rows, cols = x.shape
    ldb_w = nwords(cols) if ldb_w is None else int(ldb_w)
    bits = torch.empty((rows, ldb_w), dtype=_BITS, device=x.device)
    with _on(x):
        _check(load().bnn_pack_u8(_ptr(x), int(thr), _ptr(bits), ctypes.c_int64(rows), cols, ldb_w, _stream(x)), "bnn_pack_u8")
    return bits


def pack_f32(x, thr, ldb_w: int | None = None):
    _dev(x, torch.float32, None, "x"); _dev(thr, torch.float32, 1, "thr")
    cols = x.shape[-1]
    rows = x.numel() // cols
    ldb_w = nwords(cols) if ldb_w is None else int(ldb_w)
    bits = torch.empty(tuple(x.shape[:-1]) + (ldb_w,), dtype=_BITS, device=x.device)
    with _on(x):
        _check(load().bnn_pack_f32(_ptr(x), _ptr(thr), _ptr(bits), ctypes.c_int64(rows), cols, ldb_w, _stream(x)), "bnn_pack_f32")
    return bits


def tile_b(B, K: int):
    """Weights [N][ldb_w] -> the pre-tiled layout bnn_bmm_tiled reads (32-row groups, 16-byte units interleaved)."""
    _dev(B, _BITS, 2, "B")
    N, ldb = B.shape
    out = torch.empty(((N + 31) // 32 * 32, ldb), dtype=_BITS, device=B.device)
    with _on(B):
        _check(load().bnn_tile_b(_ptr(B), _ptr(out), N, int(K), ldb, _stream(B)), "bnn_tile_b")
    return out


def bmm_tiled(A, Bt, N: int, K: int, out=None):
    _dev(A, _BITS, 2, "A"); _dev(Bt, _BITS, 2, "Bt")
    M = A.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=A.device)
    with _on(A):
        _check(load().bnn_bmm_tiled(_ptr(A), _ptr(Bt), _ptr(out), M, int(N), int(K), A.shape[1], Bt.shape[1], out.shape[1],
                                    _stream(A)), "bnn_bmm_tiled")
    return out


def bmm_thr_tiled(A, Bt, thr, N: int, K: int, ldcb_w: int | None = None, out=None):
    _dev(A, _BITS, 2, "A"); _dev(Bt, _BITS, 2, "Bt"); _dev(thr, torch.int32, 1, "thr")
    M = A.shape[0]
    ldcb_w = round_up(nwords(N), 4) if ldcb_w is None else ldcb_w
    if out is None:
        out = torch.empty((M, ldcb_w), dtype=_BITS, device=A.device)
    with _on(A):
        _check(load().bnn_bmm_thr_tiled(_ptr(A), _ptr(Bt), _ptr(thr), _ptr(out), M, int(N), int(K), A.shape[1], Bt.shape[1],
                                        out.shape[1], _stream(A)), "bnn_bmm_thr_tiled")
    return out


def panels_from_rows(X, K: int):
    """Packed [rows][ldx_w] -> the K-panel layout ([ceil(K/256)][rows][8] words) that bmm_panels / bmm_thr_panels read."""
    _dev(X, _BITS, 2, "X")
    rows, ldx = X.shape
    out = torch.empty(((int(K) + 255) // 256, rows, 8), dtype=_BITS, device=X.device)
    with _on(X):
        _check(load().bnn_panels_from_rows(_ptr(X), _ptr(out), ctypes.c_int64(rows), int(K), ldx, _stream(X)), "bnn_panels_from_rows")
    return out


def rows_from_panels(Xp, K: int, ldx_w: int | None = None):
    """The K-panel layout back to packed rows [rows][ldx_w]."""
    _dev(Xp, _BITS, 3, "Xp")
    rows = Xp.shape[1]
    ldx_w = round_up(nwords(K), 4) if ldx_w is None else int(ldx_w)
    out = torch.empty((rows, ldx_w), dtype=_BITS, device=Xp.device)
    with _on(Xp):
        _check(load().bnn_rows_from_panels(_ptr(Xp), _ptr(out), ctypes.c_int64(rows), int(K), ldx_w, _stream(Xp)), "bnn_rows_from_panels")
    return out


def bmm_panels(Ap, Bp, K: int, out=None):
    """int32 [M][N] = A x B^T with both operands in K panels ([panels][rows][8])."""
    _dev(Ap, _BITS, 3, "Ap"); _dev(Bp, _BITS, 3, "Bp")
    M, N = Ap.shape[1], Bp.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=Ap.device)
    with _on(Ap):
        _check(load().bnn_bmm_panels(_ptr(Ap), _ptr(Bp), _ptr(out), M, N, int(K), out.shape[1], _stream(Ap)), "bnn_bmm_panels")
    return out


def bmm_thr_panels(Ap, Bp, thr, K: int, out=None):
    """Fused threshold; the output bits come in K panels ([ceil(N/256)][M][8]), the next product's A."""
    _dev(Ap, _BITS, 3, "Ap"); _dev(Bp, _BITS, 3, "Bp"); _dev(thr, torch.int32, 1, "thr")
    M, N = Ap.shape[1], Bp.shape[1]
    if out is None:
        out = torch.empty(((N + 255) // 256, M, 8), dtype=_BITS, device=Ap.device)
    with _on(Ap):
        _check(load().bnn_bmm_thr_panels(_ptr(Ap), _ptr(Bp), _ptr(thr), _ptr(out), M, N, int(K), _stream(Ap)), "bnn_bmm_thr_panels")
    return out


def probe_load_stride(stride_bytes: int, rows: int | None = None, iters: int = 4096, dependent: bool = True, device="cuda",
                      footprint_bytes: int = 1 << 20):
    """Shader-cycle-counter ticks per MFMA operand-fragment load of one wave, rows `stride_bytes` apart (diagnostic).
    By default the buffer is `footprint_bytes` in all, so that every stride is measured at the same cache level."""
    if rows is None:
        rows = max(32, footprint_bytes // stride_bytes // 32 * 32)
    buf = torch.zeros(rows * stride_bytes // 4, dtype=_BITS, device=device)
    cyc = torch.zeros(2, dtype=torch.int64, device=device)
    with _on(buf):
        for _ in range(2):                                  # the second run has the buffer in cache
            _check(load().bnn_probe_load_stride(_ptr(buf), _ptr(cyc), int(stride_bytes), int(rows), int(iters),
                                                1 if dependent else 0, _stream(buf)), "bnn_probe_load_stride")
    return float(cyc[0].item()) / iters


PROBES = {"mfma_fp4": 0, "mfma_fp4_expand": 1, "mfma_i8": 2, "mfma_bf16": 3, "valu_xor_popc": 4, "lds_read": 5,
          "hbm_read": 6, "hbm_write": 7, "hbm_copy": 8}


def probe_pipeline(which: str, buf, iters: int = 2000, reps: int = 3):
    """Runs one ceiling microbenchmark (bnn_probe_pipeline) `reps` times after a warm-up launch; returns
    (work units per second of the fastest launch, seconds of that launch).  buf: a uint8 device tensor."""
    _dev(buf, torch.uint8, 1, "buf")
    work = ctypes.c_double(0.0)
    best = None
    with _on(buf):
        for rep in range(reps + 1):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            _check(load().bnn_probe_pipeline(PROBES[which], _ptr(buf), ctypes.c_size_t(buf.numel()), int(iters),
                                             ctypes.byref(work), _stream(buf)), "bnn_probe_pipeline")
            e1.record()
            e1.synchronize()
            sec = e0.elapsed_time(e1) * 1e-3
            if rep > 0 and (best is None or sec < best):
                best = sec
    return work.value / best, best


def probe_pipeline_enqueue(which: str, buf, iters: int) -> float:
    """Enqueues one launch of a ceiling microbenchmark without waiting for it; returns its work units."""
    _dev(buf, torch.uint8, 1, "buf")
    work = ctypes.c_double(0.0)
    with _on(buf):
        _check(load().bnn_probe_pipeline(PROBES[which], _ptr(buf), ctypes.c_size_t(buf.numel()), int(iters),
                                         ctypes.byref(work), _stream(buf)), "bnn_probe_pipeline")
    return work.value


def sign_pack_f32(x, ldb_w: int | None = None):
    """Binarization by sign: x [rows][cols] fp32 -> bits [rows][ldb_w], bit = (x >= 0)."""
    _dev(x, torch.float32, 2, "x")
    rows, cols = x.shape
    ldb_w = nwords(cols) if ldb_w is None else ldb_w
    bits = torch.empty((rows, ldb_w), dtype=_BITS, device=x.device)
    with _on(x):
        _check(load().bnn_sign_pack_f32(_ptr(x), _ptr(bits), ctypes.c_int64(rows), cols, cols, ldb_w, _stream(x)), "bnn_sign_pack_f32")
    return bits


def bmm_general_f32(A, B, out=None, workspace=None):
    """General BMM: fp32 A [M][K], B [N][K] -> fp32 [M][N] of the sign-binarized product."""
    if out is None and workspace is None:
        done = (_native or _load_native()).bmm_general_f32(A, B)
        if done is not None:
            return done
    _dev(A, torch.float32, 2, "A"); _dev(B, torch.float32, 2, "B")
    M, K = A.shape
    N = B.shape[0]
    if B.shape[1] != K:
        raise ValueError("K mismatch")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    if workspace is None:
        workspace = torch.empty(max(int(load().bnn_bmm_general_workspace_bytes(M, N, K)), 256), dtype=torch.uint8, device=A.device)
    with _on(A):
        _check(load().bnn_bmm_general_f32(_ptr(A), _ptr(B), _ptr(out), M, N, K, K, K, N, _ptr(workspace),
                                          ctypes.c_size_t(workspace.numel()), _stream(A)), "bnn_bmm_general_f32")
    return out


def bconv_general_f32(x, filt, stride: int, pad: int, pad_mode: int = PAD_MINUS_ONE, out=None, workspace=None):
    """General BConv: fp32 x [N][H][W][C], filt [O][k][k][C] -> fp32 [N][P][Q][O] of the sign-binarized convolution."""
    _dev(x, torch.float32, 4, "x"); _dev(filt, torch.float32, 4, "filt")
    N, H, W, C = x.shape
    O, k, _, C2 = filt.shape
    if C != C2:
        raise ValueError("channel mismatch")
    P = (H + 2 * pad - k) // stride + 1 if stride > 0 else 1
    Q = (W + 2 * pad - k) // stride + 1 if stride > 0 else 1
    if out is None:
        out = torch.empty((N, max(P, 1), max(Q, 1), O), dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(max(int(load().bnn_bconv_general_workspace_bytes(N, H, W, C, O, k)), 256), dtype=torch.uint8,
                                device=x.device)
    with _on(x):
        _check(load().bnn_bconv_general_f32(_ptr(x), _ptr(filt), _ptr(out), N, H, W, C, O, k, int(stride), int(pad), int(pad_mode),
                                            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(x)), "bnn_bconv_general_f32")
    return out


def unpack_i32(bits, cols: int):
    _dev(bits, _BITS, None, "bits")
    ldb_w = bits.shape[-1]
    rows = bits.numel() // ldb_w
    out = torch.empty(tuple(bits.shape[:-1]) + (cols,), dtype=torch.int32, device=bits.device)
    with _on(bits):
        _check(load().bnn_unpack_i32(_ptr(bits), _ptr(out), ctypes.c_int64(rows), int(cols), ldb_w, int(cols), _stream(bits)),
               "bnn_unpack_i32")
    return out


def maxpool_or(bits, C: int, win: int, stride: int):
    """bits [N][H][W][cw] -> [N][P][Q][cw]: max-pooling of +1/-1 activations as a bitwise OR."""
    done = (_native or _load_native()).maxpool_or(bits, C, win, stride)
    if done is not None:
        return done
    _dev(bits, _BITS, 4, "bits")
    N, H, W, cw = bits.shape
    ok = stride >= 1 and 1 <= win <= min(H, W)          # anything else is left for the library to reject
    P, Q = ((H - win) // stride + 1, (W - win) // stride + 1) if ok else (1, 1)
    out = torch.empty((N, P, Q, cw), dtype=_BITS, device=bits.device)
    with _on(bits):
        _check(load().bnn_maxpool_or(_ptr(bits), _ptr(out), N, H, W, int(C), int(win), int(stride), _stream(bits)),
               "bnn_maxpool_or")
    return out


def conv_f32_thr(x, w, thr, stride: int, pad: int, want_f32: bool = False):
    """fp32 first layer: x [N][H][W][C], w [O][k][k][C], thr [O] -> bits [N][P][Q][ow] (and fp32 y)."""
    _dev(x, torch.float32, 4, "x"); _dev(w, torch.float32, 4, "w"); _dev(thr, torch.float32, 1, "thr")
    N, H, W, C = x.shape
    O, k, _, C2 = w.shape
    if C != C2:
        raise ValueError("channel mismatch")
    P = (H + 2 * pad - k) // stride + 1
    Q = (W + 2 * pad - k) // stride + 1
    bits = torch.empty((N, P, Q, nwords(O)), dtype=_BITS, device=x.device)
    y = torch.empty((N, P, Q, O), dtype=torch.float32, device=x.device) if want_f32 else None
    with _on(x):
        _check(load().bnn_conv_f32_thr(_ptr(x), _ptr(w), _ptr(thr), _ptr(y), _ptr(bits), N, H, W, C, O, k, int(stride), int(pad),
                                       _stream(x)), "bnn_conv_f32_thr")
    return (bits, y) if want_f32 else bits


def conv_f32_split_thr(x, w, thr, stride: int, pad: int, want_f32: bool = False, workspace=None, products: int = 9):
    """fp32 first layer on the bf16 matrix cores (inputs and weights split exactly into three bf16 terms each;
    products: 9 term products, or 6 without the three smallest)."""
    if workspace is None and want_f32 is False:
        done = (_native or _load_native()).conv_f32_split_thr(x, w, thr, stride, pad, products)
        if done is not None:
            return done
    _dev(x, torch.float32, 4, "x"); _dev(w, torch.float32, 4, "w"); _dev(thr, torch.float32, 1, "thr")
    N, H, W, C = x.shape
    O, k, _, C2 = w.shape
    if C != C2:
        raise ValueError("channel mismatch")
    P = (H + 2 * pad - k) // stride + 1
    Q = (W + 2 * pad - k) // stride + 1
    bits = torch.empty((N, P, Q, nwords(O)), dtype=_BITS, device=x.device)
    y = torch.empty((N, P, Q, O), dtype=torch.float32, device=x.device) if want_f32 else None
    if workspace is None:
        workspace = torch.empty(max(int(load().bnn_conv_f32_split_workspace_bytes(C, O, k)), 16), dtype=torch.uint8, device=x.device)
    with _on(x):
        _check(load().bnn_conv_f32_split_thr_ex(_ptr(x), _ptr(w), _ptr(thr), _ptr(y), _ptr(bits), N, H, W, C, O, k, int(stride),
                                                int(pad), int(products), _ptr(workspace), ctypes.c_size_t(workspace.numel()),
                                                _stream(x)), "bnn_conv_f32_split_thr_ex")
    return (bits, y) if want_f32 else bits


def bwn_conv_thr(x, wbits, thr, C: int, stride: int, pad: int, want_f32: bool = False, workspace=None):
    """First layer with binarized weights: x [N][H][W][C] fp32, wbits [O][k][k][cw], thr [O] -> bits (and fp32 y)."""
    if workspace is None and want_f32 is False:
        done = (_native or _load_native()).bwn_conv_thr(x, wbits, thr, C, stride, pad)
        if done is not None:
            return done
    _dev(x, torch.float32, 4, "x"); _dev(wbits, _BITS, 4, "wbits"); _dev(thr, torch.float32, 1, "thr")
    N, H, W, C2 = x.shape
    O, k, _, cw = wbits.shape
    if C != C2 or cw != nwords(C):
        raise ValueError("channel mismatch")
    P = (H + 2 * pad - k) // stride + 1
    Q = (W + 2 * pad - k) // stride + 1
    bits = torch.empty((N, P, Q, nwords(O)), dtype=_BITS, device=x.device)
    y = torch.empty((N, P, Q, O), dtype=torch.float32, device=x.device) if want_f32 else None
    if workspace is None:
        workspace = torch.empty(max(int(load().bnn_bwn_workspace_bytes(C, O, k)), 16), dtype=torch.uint8, device=x.device)
    with _on(x):
        _check(load().bnn_bwn_conv_thr(_ptr(x), _ptr(wbits), _ptr(thr), _ptr(y), _ptr(bits), N, H, W, C, O, k, int(stride), int(pad),
                                       _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(x)), "bnn_bwn_conv_thr")
    return (bits, y) if want_f32 else bits


def head_f32(bits, w, C: int, want_pooled: bool = False):
    """bits [N][H][W][cw] -> fp32 logits [N][J] = FC(sum-pool(+1/-1) / HW); w [J][C]."""
    _dev(bits, _BITS, 4, "bits"); _dev(w, torch.float32, 2, "w")
    N, H, W, cw = bits.shape
    J = w.shape[0]
    y = torch.empty((N, J), dtype=torch.float32, device=bits.device)
    pooled = torch.empty((N, C), dtype=torch.int32, device=bits.device) if want_pooled else None
    with _on(bits):
        _check(load().bnn_head_f32(_ptr(bits), _ptr(w), _ptr(y), _ptr(pooled), N, H * W, int(C), J, _stream(bits)), "bnn_head_f32")
    return (y, pooled) if want_pooled else y


_TYPE_CODE = {torch.uint8: 0, torch.int32: 1, torch.float32: 2}          # as the native module counts them


class Net:
    """Layer-chained forward (bnn_net_*).  Keeps references to every weight tensor it borrows."""

    def __init__(self):
        self._h = ctypes.c_void_p()
        _check(load().bnn_net_create(ctypes.byref(self._h)), "bnn_net_create")
        self._keep = []
        self._ws = None
        self._out_kind = None
        self._out_cols = 0
        self.n_layers = 0

    def __del__(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            load().bnn_net_destroy(self._h)
            self._h = ctypes.c_void_p()

    def _added(self, *tensors):
        self._keep.extend(t for t in tensors if t is not None)
        self.n_layers += 1

    def input_u8(self, cols: int, thr: int):
        _check(load().bnn_net_input_u8(self._h, int(cols), int(thr)), "bnn_net_input_u8")
        self._in_dtype = torch.uint8
        self._added()

    def input_bits(self, cols: int):
        _check(load().bnn_net_input_bits(self._h, int(cols)), "bnn_net_input_bits")
        self._in_dtype = _BITS
        self._added()

    def input_conv_f32(self, w, thr, H: int, W: int, stride: int, pad: int):
        _dev(w, torch.float32, 4, "w"); _dev(thr, torch.float32, 1, "thr")
        O, k, _, C = w.shape
        _check(load().bnn_net_input_conv_f32(self._h, _ptr(w), _ptr(thr), int(H), int(W), C, O, k, int(stride), int(pad)),
               "bnn_net_input_conv_f32")
        self._in_dtype = torch.float32
        self._added(w, thr)

    def input_bwn_f32(self, wbits, thr, H: int, W: int, C: int, stride: int, pad: int):
        _dev(wbits, _BITS, 4, "wbits"); _dev(thr, torch.float32, 1, "thr")
        O, k, _, cw = wbits.shape
        if cw != nwords(C):
            raise ValueError("channel mismatch")
        _check(load().bnn_net_input_bwn_f32(self._h, _ptr(wbits), _ptr(thr), int(H), int(W), int(C), O, k, int(stride), int(pad)),
               "bnn_net_input_bwn_f32")
        self._in_dtype = torch.float32
        self._added(wbits, thr)

    def add_fc(self, W, thr, K: int):
        _dev(W, _BITS, 2, "W")
        if thr is not None:
            _dev(thr, torch.int32, 1, "thr")
        N = W.shape[0]
        if W.shape[1] != round_up(nwords(K), 4):
            raise ValueError("W rows must be ceil(K/32) words rounded up to a multiple of 4 (%d), got %d"
                             % (round_up(nwords(K), 4), W.shape[1]))
        _check(load().bnn_net_add_fc(self._h, _ptr(W), _ptr(thr), int(K), N), "bnn_net_add_fc")
        if thr is None:
            self._out_kind, self._out_cols = torch.int32, N
        self._added(W, thr)

    def add_conv(self, filt, thr, C: int, stride: int, pad: int, pad_mode: int = PAD_MINUS_ONE):
        _dev(filt, _BITS, 4, "filt"); _dev(thr, torch.int32, 1, "thr")
        O, k = filt.shape[0], filt.shape[1]
        _check(load().bnn_net_add_conv(self._h, _ptr(filt), _ptr(thr), int(C), O, k, int(stride), int(pad), int(pad_mode)),
               "bnn_net_add_conv")
        self._added(filt, thr)

    def add_pool(self, win: int, stride: int):
        _check(load().bnn_net_add_pool(self._h, int(win), int(stride)), "bnn_net_add_pool")
        self._added()

    def add_block(self, W1, thr1, W2, thr2, Wd, cin: int, cout: int, stride: int, pad_mode: int = PAD_MINUS_ONE):
        for t in (W1, W2):
            _dev(t, _BITS, 4, "W")
        _check(load().bnn_net_add_block(self._h, _ptr(W1), _ptr(thr1), _ptr(W2), _ptr(thr2), _ptr(Wd), int(cin), int(cout),
                                        int(stride), int(pad_mode)), "bnn_net_add_block")
        self._added(W1, thr1, W2, thr2, Wd)

    def add_head_f32(self, w):
        _dev(w, torch.float32, 2, "w")
        _check(load().bnn_net_add_head_f32(self._h, _ptr(w), w.shape[0]), "bnn_net_add_head_f32")
        self._out_kind, self._out_cols = torch.float32, w.shape[0]
        self._added(w)

    @classmethod
    def from_layers(cls, layers, in_hw: int, device="cuda"):
        """Builds a net from a list of layer dicts holding numpy arrays (the description the seeded
        generators and the CPU oracle use): conv_f32 first, then bconv / pool / block / fc."""
        import numpy as np

        def dev(a):
            a = np.ascontiguousarray(a)
            return torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).to(device)

        net = cls()
        for L in layers:
            op = L["op"]
            if op == "conv_f32":
                net.input_conv_f32(dev(L["w"]), dev(L["thr"]), in_hw, in_hw, L["stride"], L["pad"])
            elif op == "bwn":
                net.input_bwn_f32(dev(L["W"]), dev(L["thr"]), in_hw, in_hw, L["C"], L["stride"], L["pad"])
            elif op == "bconv":
                net.add_conv(dev(L["W"]), dev(L["thr"]), L["C"], L["stride"], L["pad"])
            elif op == "pool":
                net.add_pool(L["win"], L["stride"])
            elif op == "block":
                net.add_block(dev(L["W1"]), dev(L["thr1"]), dev(L["W2"]), dev(L["thr2"]),
                              dev(L["Wd"]) if "Wd" in L else None, L["cin"], L["cout"], L["stride"])
            elif op == "fc":
                net.add_fc(dev(L["W"]), None if L["thr"] is None else dev(L["thr"]), L["K"])
            else:
                raise ValueError(op)
        return net

    def workspace_bytes(self, batch: int) -> int:
        n = ctypes.c_size_t()
        _check(load().bnn_net_workspace_bytes(self._h, int(batch), ctypes.byref(n)), "bnn_net_workspace_bytes")
        return n.value

    def fc_run(self, batch: int, recorded: bool = False) -> int:
        """How many layers at the head of the net forward() runs as one launch (0: each by itself); recorded: under graph capture."""
        n = ctypes.c_int()
        _check(load().bnn_net_fc_run(self._h, int(batch), int(recorded), ctypes.byref(n)), "bnn_net_fc_run")
        return n.value

    def forward(self, x, out=None, path: int = PATH_AUTO):
        if out is None and self._ws is not None and self._out_kind is not None:
            done = (_native or _load_native()).net_forward(self._h.value, x, _TYPE_CODE[self._in_dtype], self._ws, self._out_cols,
                                                           _TYPE_CODE[self._out_kind], path)
            if done is not None:
                return done
        _dev(x, self._in_dtype, None, "input")
        batch = x.shape[0]
        need = self.workspace_bytes(batch)
        if self._ws is None or self._ws.numel() < need or self._ws.device != x.device:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
        if out is None:
            out = torch.empty((batch, self._out_cols), dtype=self._out_kind, device=x.device)
        with _on(x):
            _check(load().bnn_net_forward(self._h, _ptr(x), _ptr(out), batch, _ptr(self._ws), ctypes.c_size_t(self._ws.numel()),
                                          int(path), _stream(x)), "bnn_net_forward")
        return out

    def forward_static(self, x, out=None, path: int = PATH_AUTO):
        """bnn_net_forward_static: the same forward on the library's fixed per-GPU workspace (no allocation inside
        the library; the output tensor must be passed in for a call that allocates nothing at all)."""
        _dev(x, self._in_dtype, None, "input")
        batch = x.shape[0]
        if out is None:
            out = torch.empty((batch, self._out_cols), dtype=self._out_kind, device=x.device)
        with _on(x):
            _check(load().bnn_net_forward_static(self._h, _ptr(x), _ptr(out), batch, int(path), _stream(x)),
                   "bnn_net_forward_static")
        return out

    def persistent_status(self, device=None) -> bool:
        """True if the last forward_persistent gave up at a barrier (its output is then undefined).  Waits for the
        current stream."""
        aborted = ctypes.c_int(-1)
        dev = self._ws.device if device is None else device
        with torch.cuda.device(dev):
            _check(load().bnn_net_persistent_status(self._h, ctypes.byref(aborted),
                                                    ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)),
                   "bnn_net_persistent_status")
        return aborted.value != 0

    def forward_persistent(self, x, out=None, no_sync: bool = False, give_up_at_once: bool = False, grid_cap: int = 0):
        """Same forward with every run of FC / 3x3 convolution / residual-block layers as one kernel launch.  no_sync
        skips the device-wide barriers (results undefined, for timing the barriers only); give_up_at_once makes every
        barrier wait time out at its first poll (results undefined, for testing the time-out report); grid_cap > 0
        bounds the number of workgroups."""
        _dev(x, self._in_dtype, None, "input")
        batch = x.shape[0]
        need = self.workspace_bytes(batch)
        if self._ws is None or self._ws.numel() < need or self._ws.device != x.device:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
        if out is None:
            out = torch.empty((batch, self._out_cols), dtype=self._out_kind, device=x.device)
        with _on(x):
            _check(load().bnn_net_forward_persistent(self._h, _ptr(x), _ptr(out), batch, _ptr(self._ws),
                                                     ctypes.c_size_t(self._ws.numel()),
                                                     (1 if no_sync else 0) | (2 if give_up_at_once else 0) | ((int(grid_cap) & 0xFFFF) << 8),
                                                     _stream(x)),
                   "bnn_net_forward_persistent")
        return out

    def layer_bits(self, layer: int):
        """Copy of the packed bits produced by `layer` in the last forward, as [rows][words]."""
        p = ctypes.c_void_p()
        rows = ctypes.c_int64()
        wpr = ctypes.c_int()
        _check(load().bnn_net_layer_bits(self._h, int(layer), ctypes.byref(p), ctypes.byref(rows), ctypes.byref(wpr)),
               "bnn_net_layer_bits")
        off = p.value - self._ws.data_ptr()
        n = rows.value * wpr.value * 4
        return self._ws[off:off + n].view(_BITS).view(rows.value, wpr.value).clone()


class _Cache4Struct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("page", ctypes.c_int),
                ("signs", ctypes.c_int)]


class _Rows4Struct(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("start", ctypes.c_void_p), ("batch", ctypes.c_int), ("table_pages", ctypes.c_int),
                ("tokens", ctypes.c_int)]


_ELEMENTS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # BNN_F32, BNN_BF16, BNN_F16


class _RotationStruct(ctypes.Structure):
    _fields_ = [("frequencies", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("pairs", ctypes.c_int), ("neighbours", ctypes.c_int), ("inverse", ctypes.c_int),
                ("magnitude", ctypes.c_double)]


def _rotation(frequencies, positions, tokens, device, interleaved, inverse, magnitude):
    _dev(frequencies, torch.float64, 1, "frequencies")
    if positions is not None and _dev(positions, torch.int32, 1, "positions").shape[0] != tokens:
        raise ValueError("positions must have an entry for every token")
    for t in (frequencies, positions):
        if t is not None and t.device != device:
            raise ValueError("frequencies and positions must be on the elements' device")
    return _RotationStruct(frequencies.data_ptr(), 0 if positions is None else positions.data_ptr(), frequencies.shape[0], int(bool(interleaved)), int(bool(inverse)), float(magnitude))


def _distances(x):
    """Elements between tokens and between heads of x [tokens][heads][dim]; of a dimension of a single entry there are none."""
    return tuple(ctypes.c_int64(x.stride(i) if x.shape[i] > 1 else 0) for i in (0, 1))


def _heads_of(x, name):
    """x [tokens][heads][dim], the elements of a head side by side -> its type code."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("%s must be a device tensor" % name)
    if x.dtype not in _ELEMENTS:
        raise TypeError("%s must be fp32, bf16 or fp16, got %s" % (name, x.dtype))
    if x.dim() != 3:
        raise ValueError("%s must be [tokens][heads][dim]" % name)
    if x.stride(2) != 1 and x.shape[2] > 1 and x.numel() != 0:
        raise ValueError("the elements of a head of %s must be contiguous" % name)
    return _ELEMENTS[x.dtype]


def rotary_frequencies(elements: int, base: float = 10000.0, factor: float = 1.0, scaling: str = "linear", context: int = 0, low: float = 1.0, high: float = 32.0, device="cuda"):
    """Frequencies base^(-2p / elements) of elements / 2 pairs, float64 on the device, for contexts `factor` times as long as those of training:
    scaling "linear" divides them all by it; "base" raises the base by factor^(elements / (elements - 2)), so that the first keeps its value and the last is divided;
    "parts" divides those that turn less than `low` times over `context` positions, keeps those that turn more than `high` times, and blends between (with it, a
    magnitude of 1 + 0.1 ln(factor) is usual)."""
    if elements < 2 or elements % 2 or not base > 0 or not factor >= 1:
        raise ValueError("an even number of elements, base > 0 and factor >= 1 expected")
    if scaling == "base" and factor != 1:
        if elements < 4:
            raise ValueError("scaling by the base needs two pairs at least")
        base = base * factor ** (elements / (elements - 2))
    f = float(base) ** (-torch.arange(0, elements, 2, dtype=torch.float64) / elements)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if context < 1 or not high > low:
            raise ValueError("parts are told apart by context >= 1, and high > low")
        kept = ((context * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * kept + f / factor * (1 - kept)
    elif scaling != "base":
        raise ValueError("scaling is linear, base or parts")
    return f.to(device)


def rotary(x, positions, frequencies, interleaved: bool = False, magnitude: float = 1.0, inverse: bool = False, out=None):
    """x [tokens][heads][dim] (fp32, bf16 or fp16) with every head's first 2 * len(frequencies) elements turned in pairs by positions[token] * frequencies[pair]
    (positions int32, frequencies float64: rotary_frequencies); pairs are the halves' elements, or neighbours if interleaved.  inverse turns back, which is also how a
    gradient passes.  out may be x (else no part of it); no two heads of it share an element."""
    if out is None:
        done = (_native or _load_native()).rotary(x, frequencies, positions, interleaved, magnitude, inverse)
        if done is not None:
            return done
    code = _heads_of(x, "x")
    rot = _rotation(frequencies, positions, x.shape[0], x.device, interleaved, inverse, magnitude)
    if positions is None:
        raise TypeError("positions must be a device tensor")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _heads_of(out, "out")
        if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device:
            raise ValueError("out must have x's shape, type and device")
    with _on(x):
        _check(load().bnn_rotary(_ptr(x), _ptr(out), code, x.shape[0], x.shape[1], x.shape[2], *_distances(x), *_distances(out), ctypes.byref(rot), _stream(x)), "bnn_rotary")
    return out


class Cache4:
    """Key/value cache in 4 bits (bnn_cache4_*): pages of `page` tokens, a page table per batch, E2M1 codes with a power of two per 32 elements.

    ``data`` (uint8 [pages][kv_heads][record]) is the cache's memory, allocated here unless given; the layout is in include/bnn.h.
    Every call takes the plan of a batch: ``table`` int32 [batch][pages of the longest], ``lens`` int32 [batch], tokens per sequence including
    those of this call, and, where sequences contribute different numbers of rows, ``start`` int32 [batch + 1].  The rows of a sequence are
    its newest tokens.  Tensors of elements are fp32, bf16 or fp16.  No call has a gradient: results of tensors that require one do not."""

    def __init__(self, pages: int | None = None, *, kv_heads: int, head_dim: int, page: int = 64, signs: bool = True, data=None, device="cuda"):
        record = int(load().bnn_cache4_record_bytes(int(head_dim), int(page), int(bool(signs))))
        if record == 0:
            raise ValueError("head_dim of 64, 96, 128, 192 or 256 and pages of 16 to 256 tokens, a power of two, expected")
        if data is None:
            if pages is None:
                raise ValueError("pages or data expected")
            data = torch.empty((int(pages), int(kv_heads), record), dtype=torch.uint8, device=device)
        _dev(data, torch.uint8, 3, "data")
        if data.shape[1] != kv_heads or data.shape[2] != record or pages not in (None, data.shape[0]):
            raise ValueError("data must be [pages][kv_heads][%d]" % record)
        self.kv_heads, self.head_dim, self.page, self.signs = int(kv_heads), int(head_dim), int(page), bool(signs)
        self._plain = (data, self.kv_heads, self.head_dim, self.page, int(self.signs))         # what the native module takes

    @property
    def data(self):
        return self._plain[0]

    def _struct(self):
        return ctypes.byref(_Cache4Struct(self.data.data_ptr(), self.data.shape[0], self.kv_heads, self.head_dim, self.page, int(self.signs)))

    def _rows(self, table, lens, start, tokens):
        _dev(table, torch.int32, 2, "table"); _dev(lens, torch.int32, 1, "lens")
        batch, width = table.shape
        if lens.shape[0] != batch:
            raise ValueError("lens must have an entry for every sequence of table")
        if start is not None and _dev(start, torch.int32, 1, "start").shape[0] != batch + 1:
            raise ValueError("start must have one entry more than table has sequences")
        for t in (table, lens, start):
            if t is not None and t.device != self.data.device:
                raise ValueError("the plan must be on the cache's device")
        return _Rows4Struct(table.data_ptr(), lens.data_ptr(), 0 if start is None else start.data_ptr(), batch, width, int(tokens))

    def _elements(self, x, heads, name):
        """Type code and distances of x [tokens][heads][head_dim]; only the elements of a head need be contiguous."""
        if not isinstance(x, torch.Tensor) or not x.is_cuda:
            raise TypeError("%s must be a device tensor" % name)
        if x.dtype not in _ELEMENTS:
            raise TypeError("%s must be fp32, bf16 or fp16, got %s" % (name, x.dtype))
        if x.dim() != 3 or x.shape[2] != self.head_dim or (heads is not None and x.shape[1] != heads):
            raise ValueError("%s must be [tokens][%s][%d]" % (name, "heads" if heads is None else heads, self.head_dim))
        if x.device != self.data.device:
            raise ValueError("%s must be on the cache's device" % name)
        if x.stride(2) != 1 and x.numel() != 0:
            raise ValueError("the elements of a head of %s must be contiguous" % name)
        return _ELEMENTS[x.dtype], *(ctypes.c_int64(x.stride(i) if x.shape[i] > 1 else 0) for i in (0, 1))

    def _workspace(self, workspace):
        """The caller's: plain bytes on the cache's device (that they suffice is checked by the library)."""
        if _dev(workspace, torch.uint8, 1, "workspace").device != self.data.device:
            raise ValueError("workspace must be on the cache's device")
        return workspace

    def write(self, k, v, table, lens, start=None):
        """Quantises k, v [tokens][kv_heads][head_dim], the newest tokens of every sequence, into the cache."""
        if (_native or _load_native()).cache4_write(*self._plain, table, lens, start, k, v):
            return
        code, kt, kh = self._elements(k, self.kv_heads, "k")
        code_v, vt, vh = self._elements(v, self.kv_heads, "v")
        if code != code_v or k.shape != v.shape:
            raise ValueError("k and v must agree in type and shape")
        rows = self._rows(table, lens, start, k.shape[0])
        with _on(k):
            _check(load().bnn_cache4_write(self._struct(), ctypes.byref(rows), _ptr(k), _ptr(v), code, kt, kh, vt, vh, _stream(k)), "bnn_cache4_write")

    def write_rotary(self, q, k, v, table, lens, frequencies, start=None, positions=None, interleaved: bool = False, magnitude: float = 1.0, out=None):
        """write() of v and of k turned by its tokens' positions, as rotary() does it; returns q [tokens][heads][head_dim] turned alike, or None without q.  positions (int32
        [tokens]): by default a token's place in its sequence, which is no longer its position once tokens before it were evicted."""
        if out is None and q is not None:
            done = (_native or _load_native()).cache4_write_rotary(*self._plain, table, lens, start, q, k, v, frequencies, positions, interleaved, magnitude, False)
            if done is not None:
                return done
        code, kt, kh = self._elements(k, self.kv_heads, "k")
        code_v, vt, vh = self._elements(v, self.kv_heads, "v")
        if code != code_v or k.shape != v.shape:
            raise ValueError("k and v must agree in type and shape")
        qt = qh = ctypes.c_int64(0)
        if q is not None:
            code_q, qt, qh = self._elements(q, None, "q")
            if code_q != code or q.shape[0] != k.shape[0]:
                raise ValueError("q must have k's type and tokens")
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            elif _dev(out, q.dtype, 3, "out").shape != q.shape or out.device != q.device:
                raise ValueError("out must have q's shape and device")
        elif out is not None:
            raise ValueError("out without q")
        rows = self._rows(table, lens, start, k.shape[0])
        rot = _rotation(frequencies, positions, k.shape[0], k.device, interleaved, False, magnitude)
        with _on(k):
            _check(load().bnn_cache4_write_rotary(self._struct(), ctypes.byref(rows), ctypes.byref(rot), _ptr(q), qt, qh, 0 if q is None else q.shape[1], _ptr(out), _ptr(k), _ptr(v),
                                                  code, kt, kh, vt, vh, _stream(k)), "bnn_cache4_write_rotary")
        return out

    def read(self, table, lens, start=None, tokens: int | None = None, dtype=torch.bfloat16):
        """(k, v) [tokens][kv_heads][head_dim]: the newest tokens of every sequence as the cache holds them.  tokens: rows in all (default: one of every sequence)."""
        if dtype not in _ELEMENTS:
            raise TypeError("fp32, bf16 or fp16 expected, got %s" % dtype)
        tokens = table.shape[0] if tokens is None else int(tokens)
        done = (_native or _load_native()).cache4_read(*self._plain, table, lens, start, tokens, _ELEMENTS[dtype])
        if done is not None:
            return done
        rows = self._rows(table, lens, start, tokens)
        k, v = (torch.empty((tokens, self.kv_heads, self.head_dim), dtype=dtype, device=self.data.device) for _ in range(2))
        with _on(k):
            _check(load().bnn_cache4_read(self._struct(), ctypes.byref(rows), _ptr(k), _ptr(v), _ELEMENTS[dtype], _stream(k)), "bnn_cache4_read")
        return k, v

    def select(self, q, table, lens, keep: int, start=None, first: int = 1, last: int = 1, workspace=None):
        """int32 [tokens][kv_heads][keep]: the blocks (pages of a sequence) that every row of q [tokens][heads][head_dim] attends to, by the
        agreement of sign bits; the first `first` and the `last` most recent always; ascending, the rest -1."""
        if workspace is None:
            done = (_native or _load_native()).cache4_select(*self._plain, table, lens, start, q, keep, first, last)
            if done is not None:
                return done
        code, qt, qh = self._elements(q, None, "q")
        rows = self._rows(table, lens, start, q.shape[0])
        blocks = torch.empty((q.shape[0], self.kv_heads, max(int(keep), 0)), dtype=torch.int32, device=q.device)
        if workspace is None:
            need = int(load().bnn_cache4_select_workspace_bytes(self._struct(), ctypes.byref(rows)))
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
        else:
            self._workspace(workspace)
        with _on(q):
            _check(load().bnn_cache4_select(self._struct(), ctypes.byref(rows), _ptr(q), code, qt, qh, q.shape[1], int(keep), int(first), int(last),
                                            _ptr(blocks), _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream(q)), "bnn_cache4_select")
        return blocks

    def attend(self, q, table, lens, start=None, scale: float | None = None, causal: bool = True, window: int = 0, blocks=None, want_lse: bool = False,
               out=None, workspace=None):
        """Attention of q [tokens][heads][head_dim], the newest tokens of every sequence, over the cache -> [tokens][heads][head_dim] of q's type (and
        the logarithm of the weights' sum, fp32 [tokens][heads]).  blocks: only those (from select).  scale: 1 / sqrt(head_dim) by default."""
        scale = self.head_dim ** -0.5 if scale is None else float(scale)
        if out is None and workspace is None:
            done = (_native or _load_native()).cache4_attend(*self._plain, table, lens, start, q, scale, causal, window, blocks, want_lse)
            if done is not None:
                return done
        code, qt, qh = self._elements(q, None, "q")
        rows = self._rows(table, lens, start, q.shape[0])
        keep = 0
        if blocks is not None:
            _dev(blocks, torch.int32, 3, "blocks")
            keep = blocks.shape[2]
            if blocks.shape[0] != q.shape[0] or blocks.shape[1] != self.kv_heads or keep < 1 or blocks.device != q.device:
                raise ValueError("blocks must be [tokens][kv_heads][keep], keep >= 1, on q's device")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif _dev(out, q.dtype, 3, "out").shape != q.shape or out.device != q.device:
            raise ValueError("out must have q's shape and device")
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
        if workspace is None:
            need = int(load().bnn_cache4_attend_workspace_bytes(self._struct(), ctypes.byref(rows), code, q.shape[1], int(window), keep))
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        else:
            self._workspace(workspace)
        with _on(q):
            _check(load().bnn_cache4_attend(self._struct(), ctypes.byref(rows), _ptr(q), code, qt, qh, q.shape[1], ctypes.c_float(scale),
                                            int(bool(causal)), int(window), _ptr(blocks), keep, _ptr(out), _ptr(lse), _ptr(workspace),
                                            ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream(q)), "bnn_cache4_attend")
        return (out, lse) if want_lse else out

    def _weights(self, weights, batch, room, name):
        """fp32 [batch][kv_heads][at least the table's tokens], on the cache's device."""
        _dev(weights, torch.float32, 3, name)
        if weights.shape[0] != batch or weights.shape[1] != self.kv_heads or weights.shape[2] < room:
            raise ValueError("%s must be [batch][kv_heads][tokens], with room for the table's %d" % (name, room))
        if weights.device != self.data.device:
            raise ValueError("%s must be on the cache's device" % name)
        return weights

    def weigh(self, q, lse, table, lens, start=None, scale: float | None = None, causal: bool = True, window: int = 0, previous=None, decay: float = 1.0, out=None,
              workspace=None):
        """The attention weight of every cached token: decay * previous plus what the rows of q give it, with the lse that attend() of the same arguments (without blocks)
        returned -> fp32 [batch][kv_heads][tokens of the table].  Tokens of this call have no previous weight.  What lies behind a sequence's end is not written (and undefined in an
        output that is made here).  out may be previous."""
        scale = self.head_dim ** -0.5 if scale is None else float(scale)
        if workspace is None:
            done = (_native or _load_native()).cache4_weigh(*self._plain, table, lens, start, q, lse, scale, causal, window, previous, decay, out)
            if done is not None:
                return done if out is None else out
        code, qt, qh = self._elements(q, None, "q")
        if q.shape[0] == 0:
            raise ValueError("weights change with the rows of a call: q must have one")
        rows = self._rows(table, lens, start, q.shape[0])
        if _dev(lse, torch.float32, 2, "lse").shape != q.shape[:2] or lse.device != q.device:
            raise ValueError("lse must be [tokens][heads], on q's device")
        batch, room = table.shape[0], table.shape[1] * self.page
        if out is None:
            out = torch.empty((batch, self.kv_heads, room) if previous is None else previous.shape, dtype=torch.float32, device=q.device)
        self._weights(out, batch, room, "out")
        if previous is not None and self._weights(previous, batch, room, "previous").shape != out.shape:
            raise ValueError("previous and out must agree in shape")
        if workspace is None:
            need = int(load().bnn_cache4_weigh_workspace_bytes(self._struct(), ctypes.byref(rows), code, q.shape[1]))
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        else:
            self._workspace(workspace)
        with _on(q):
            _check(load().bnn_cache4_weigh(self._struct(), ctypes.byref(rows), _ptr(q), code, qt, qh, q.shape[1], _ptr(lse), ctypes.c_float(scale), int(bool(causal)), int(window),
                                           _ptr(previous), ctypes.c_float(decay), _ptr(out), ctypes.c_int64(out.shape[2]), _ptr(workspace),
                                           ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream(q)), "bnn_cache4_weigh")
        return out

    def heaviest(self, weights, table, lens, keep: int, first: int = 0, last: int = 0, workspace=None):
        """(int32 [batch][kv_heads][keep], int32 [batch]): the tokens of every sequence to keep, ascending, the rest -1, and how many: all of a sequence of up to `keep`, else
        the first `first`, the last `last` and those with the largest weights.  Ties go to the lower token."""
        if workspace is None:
            done = (_native or _load_native()).cache4_heaviest(*self._plain, weights, table, lens, keep, first, last)
            if done is not None:
                return done
        _dev(table, torch.int32, 2, "table"); _dev(lens, torch.int32, 1, "lens")
        batch, width = table.shape
        if lens.shape[0] != batch:
            raise ValueError("lens must have an entry for every sequence of table")
        if table.device != self.data.device or lens.device != self.data.device:
            raise ValueError("the plan must be on the cache's device")
        self._weights(weights, batch, width * self.page, "weights")
        if int(keep) < 1:
            raise ValueError("keep >= 1 expected")
        tokens = torch.empty((batch, self.kv_heads, int(keep)), dtype=torch.int32, device=weights.device)
        kept = torch.empty(batch, dtype=torch.int32, device=weights.device)
        if workspace is None:
            need = int(load().bnn_cache4_heaviest_workspace_bytes(self._struct(), batch, width))
            workspace = torch.empty(need, dtype=torch.uint8, device=weights.device) if need else None
        else:
            self._workspace(workspace)
        with _on(weights):
            _check(load().bnn_cache4_heaviest(self._struct(), _ptr(table), _ptr(lens), batch, width, _ptr(weights), ctypes.c_int64(weights.shape[2]), int(keep), int(first), int(last),
                                              _ptr(tokens), _ptr(kept), _ptr(workspace), ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream(weights)), "bnn_cache4_heaviest")
        return tokens, kept

    def move(self, tokens, table, into, weights=None):
        """Copies token tokens[b][h][i] (from heaviest) of the sequence in table[b] to token i of the one in into[b] (int32 [batch][pages], other pages than the table's), for every kv
        head; with weights returns them moved alike, fp32 [batch][kv_heads][tokens of into], 0 where there is none, or one on no page.  The sequence's length is then heaviest's second result."""
        if weights is not None:
            done = (_native or _load_native()).cache4_move(*self._plain, tokens, table, into, weights)
            if done is not None:
                return done
        _dev(tokens, torch.int32, 3, "tokens"); _dev(table, torch.int32, 2, "table"); _dev(into, torch.int32, 2, "into")
        batch = table.shape[0]
        if tokens.shape[0] != batch or into.shape[0] != batch or tokens.shape[1] != self.kv_heads or tokens.shape[2] < 1:
            raise ValueError("tokens [batch][kv_heads][keep], keep >= 1, and into [batch][pages] expected")
        for t in (tokens, table, into):
            if t.device != self.data.device:
                raise ValueError("the plan must be on the cache's device")
        moved = None
        if weights is not None:
            self._weights(weights, batch, 1, "weights")
            moved = torch.empty((batch, self.kv_heads, into.shape[1] * self.page), dtype=torch.float32, device=weights.device)
        if moved is not None and moved.numel() == 0:
            return moved
        with _on(tokens):
            _check(load().bnn_cache4_move(self._struct(), _ptr(tokens), tokens.shape[2], _ptr(table), table.shape[1], _ptr(into), into.shape[1], batch, _ptr(weights),
                                          ctypes.c_int64(0 if weights is None else weights.shape[2]), _ptr(moved), _stream(tokens)), "bnn_cache4_move")
        return moved


TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprobs entropy lse top_logprobs top_tokens")
_LOGITS = {**_ELEMENTS, torch.int32: 3}                                  # BNN_I32


def token_logprobs(logits, targets=None, scale: float = 1.0, top: int = 0, workspace=None):
    """What rows of logits [rows][cols] (fp32, bf16, fp16, or int32 sums as bmm gives them), times scale, say of tokens: TokenLogprobs of fp32 [rows] logprobs of the targets (int64
    [rows]; 0 for one outside the columns; None without targets), entropy, lse, and the `top` (64 at most) best alternatives' logprobs and columns (int32) [rows][top], ties to
    the lower column.  A row without a distribution (all -infinity, a NaN, +infinity) gets NaN and columns of -1."""
    if workspace is None and targets is not None:
        done = (_native or _load_native()).token_logprobs(logits, targets, scale, top)
        if done is not None:
            return TokenLogprobs(*done)
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a device tensor")
    if logits.dtype not in _LOGITS:
        raise TypeError("logits must be fp32, bf16, fp16 or int32, got %s" % logits.dtype)
    if logits.dim() != 2 or logits.shape[1] < 1 or (logits.stride(1) != 1 and logits.shape[1] > 1 and logits.shape[0] > 0):
        raise ValueError("logits must be [rows][cols], the columns of a row contiguous")
    rows, cols = logits.shape
    if targets is not None and (_dev(targets, torch.int64, 1, "targets").shape[0] != rows or targets.device != logits.device):
        raise ValueError("targets must have an entry for every row, on the logits' device")
    ld, code = (logits.stride(0) if rows > 1 else 0), _LOGITS[logits.dtype]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=logits.device)
    lp, entropy, lse = (None if targets is None else new(rows)), new(rows), new(rows)
    top = int(top)
    best, tokens = new(rows, max(top, 0)), new(rows, max(top, 0), dtype=torch.int32)
    if workspace is None:
        need = int(load().bnn_token_logprobs_workspace_bytes(rows, cols, code, top))
        workspace = new(need, dtype=torch.uint8) if need else None
    elif _dev(workspace, torch.uint8, 1, "workspace").device != logits.device:
        raise ValueError("workspace must be on the logits' device")
    with _on(logits):
        _check(load().bnn_token_logprobs(_ptr(logits), code, rows, cols, ctypes.c_int64(ld), ctypes.c_float(scale), _ptr(targets), top, _ptr(lp), _ptr(entropy), _ptr(lse), _ptr(best),
                                         _ptr(tokens), _ptr(workspace), ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream(logits)), "bnn_token_logprobs")
    return TokenLogprobs(lp, entropy, lse, best, tokens)
