"""ctypes binding of libexcp.so (include/excp.h).  Argument marshalling only:
every step of compression and decompression runs in the library's CUDA kernels.
PyTorch supplies device memory and the stream.  There is no CPU fallback: if
the library cannot be loaded the import of this module's handle fails loudly."""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from dataclasses import dataclass

import torch

from . import build as _build

MEDIAN_ABS_WEIGHT = 0
MEDIAN_ABS_RESIDUAL = 1

STATUS = {0: "OK", -1: "INVALID_ARG", -2: "UNSUPPORTED", -3: "BUFFER_TOO_SMALL", -4: "CUDA",
          -5: "CORRUPT_BLOB", -6: "NONFINITE_INPUT", -7: "TIMEOUT"}

EXPORTS = ["excp_create", "excp_destroy", "excp_record_bytes", "excp_compress_bound",
           "excp_status_string", "excp_last_cuda_error", "excp_compress_tensor",
           "excp_compress_checkpoint", "excp_compress_checkpoint_indexed", "excp_compress_checkpoint_w16", "excp_decompress_checkpoint_w16",
           "excp_compress_checkpoint_host", "excp_decompress_tensor", "excp_decompress_checkpoint",
           "excp_decompress_tensor_noalloc", "excp_dense_bytes", "excp_record_to_dense", "excp_checkpoint_to_dense",
           "excp_decompress_dense_tensor", "excp_decompress_dense_checkpoint", "excp_profile_enable", "excp_profile_stage_count", "excp_profile_stage_name", "excp_profile_read",
           "excp_set_kmeans_margin", "excp_set_wait_limit", "excp_selftest_wait_timeout", "excp_set_report_sse",
           "excp_mx4_bytes", "excp_mx4_tensor_scale", "excp_mx4_quantize", "excp_mx4_dequantize", "excp_mx4_matmul", "excp_mx4_linear", "excp_mx4_linear_scratch",
           "excp_token_logprobs", "excp_token_logprobs_grad", "excp_score_status",
           "excp_act8_bytes", "excp_act8_quantize", "excp_act8_restore", "excp_act_grad_scratch", "excp_act_grad", "excp_layer_norm",
           "excp_layer_norm_grad_scratch", "excp_layer_norm_grad", "excp_linear_scratch", "excp_linear", "excp_linear_grad_input", "excp_linear_grad_weight"]


class ExcpError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: EXCP_ERR_{STATUS.get(status, status)}")
        self.status = status


class CParams(C.Structure):
    _fields_ = [("alpha", C.c_float), ("beta", C.c_float), ("bits", C.c_int), ("kmeans_iters", C.c_int),
                ("seed", C.c_ulonglong), ("median_source", C.c_int), ("flags", C.c_uint)]


class CStats(C.Structure):
    _fields_ = [("numel", C.c_ulonglong), ("nnz_w", C.c_ulonglong), ("nnz_o", C.c_ulonglong),
                ("blob_bytes", C.c_ulonglong), ("median", C.c_float), ("mean_abs_ea", C.c_float),
                ("thr_w", C.c_float), ("thr_o", C.c_float),
                ("sse_w", C.c_double), ("sse_ea", C.c_double), ("sse_eas", C.c_double)]


class CMatrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int), ("rows", C.c_size_t), ("cols", C.c_size_t), ("row_stride", C.c_size_t)]


FLAG_NO_W2M, FLAG_NO_M2W, FLAG_NO_RESIDUAL, FLAG_NO_PRUNE, FLAG_NO_QUANT = 1, 2, 4, 8, 16


@dataclass
class Params:
    alpha: float = 5e-5
    beta: float = 2.0
    bits: int = 4
    kmeans_iters: int = 10
    seed: int = 0
    median_source: int = MEDIAN_ABS_WEIGHT
    flags: int = 0          # FLAG_NO_*: the ablation switches; 0 = the full method

    def to_c(self) -> CParams:
        return CParams(self.alpha, self.beta, self.bits, self.kmeans_iters, self.seed, self.median_source,
                       self.flags)


# what the native half of the binding calls (csrc/score_binding.cpp, in the order of its table)
_SCORE_CALLS = ["excp_mx4_bytes", "excp_mx4_tensor_scale", "excp_mx4_quantize", "excp_mx4_dequantize", "excp_mx4_matmul",
                "excp_mx4_linear_scratch", "excp_mx4_linear", "excp_token_logprobs", "excp_token_logprobs_grad",
                "excp_act8_bytes", "excp_act8_quantize", "excp_act8_restore", "excp_act_grad_scratch", "excp_act_grad", "excp_layer_norm",
                "excp_layer_norm_grad_scratch", "excp_layer_norm_grad", "excp_linear_scratch", "excp_linear", "excp_linear_grad_input",
                "excp_linear_grad_weight"]
_lib = None


class _NotLoaded:
    """Stands for the native half of the binding until a scoring call asks for it."""

    def __getattr__(self, name: str):
        if name.startswith("__"):
            raise AttributeError(name)
        return getattr(load_scoring(), name)


_score = _NotLoaded()


def load_library() -> C.CDLL:
    """Loads (building first if the sources are newer) libexcp.so and declares the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build()
    lib = C.CDLL(path)
    vp, sz = C.c_void_p, C.c_size_t
    lib.excp_create.argtypes = [C.POINTER(vp), C.c_int, sz]
    lib.excp_destroy.argtypes = [vp]
    lib.excp_record_bytes.argtypes = [sz, sz, sz, C.c_int]
    lib.excp_record_bytes.restype = sz
    lib.excp_compress_bound.argtypes = [sz, C.c_int]
    lib.excp_compress_bound.restype = sz
    lib.excp_status_string.argtypes = [C.c_int]
    lib.excp_status_string.restype = C.c_char_p
    lib.excp_last_cuda_error.argtypes = [vp, C.POINTER(C.c_int)]
    lib.excp_compress_tensor.argtypes = [vp, C.POINTER(CParams), vp, vp, vp, vp, sz, vp, sz,
                                         C.POINTER(sz), C.POINTER(CStats), vp]
    lib.excp_compress_checkpoint.argtypes = [vp, C.POINTER(CParams), sz, C.POINTER(vp), C.POINTER(vp),
                                             C.POINTER(vp), C.POINTER(vp), C.POINTER(sz), vp, sz,
                                             C.POINTER(sz), C.POINTER(CStats), vp]
    lib.excp_compress_checkpoint_host.argtypes = lib.excp_compress_checkpoint.argtypes
    lib.excp_compress_checkpoint_indexed.argtypes = [vp, C.POINTER(CParams), sz, C.POINTER(vp), C.POINTER(vp),
                                                     C.POINTER(vp), C.POINTER(vp), C.POINTER(sz), C.POINTER(sz), vp, sz,
                                                     C.POINTER(sz), C.POINTER(CStats), vp]
    lib.excp_compress_checkpoint_w16.argtypes = [vp, C.POINTER(CParams), sz, C.POINTER(vp), C.POINTER(vp),
                                                 C.POINTER(vp), C.POINTER(vp), C.POINTER(sz), C.c_int, vp, sz,
                                                 C.POINTER(sz), C.POINTER(CStats), vp]
    lib.excp_decompress_checkpoint_w16.argtypes = [vp, vp, C.POINTER(sz), sz, C.POINTER(vp), C.POINTER(sz), C.c_int,
                                                   C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp]
    lib.excp_decompress_tensor.argtypes = [vp, vp, sz, vp, sz, vp, vp, vp, vp]
    lib.excp_decompress_checkpoint.argtypes = [vp, vp, C.POINTER(sz), sz, C.POINTER(vp), C.POINTER(sz),
                                               C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp]
    lib.excp_decompress_tensor_noalloc.argtypes = [vp, sz, vp, sz, vp, vp, vp, vp]
    lib.excp_dense_bytes.argtypes = [sz, C.c_int]
    lib.excp_dense_bytes.restype = sz
    lib.excp_record_to_dense.argtypes = [vp, vp, sz, sz, vp, sz, C.POINTER(sz), vp]
    lib.excp_checkpoint_to_dense.argtypes = [vp, vp, C.POINTER(sz), sz, C.POINTER(sz), vp, sz, C.POINTER(sz), vp]
    lib.excp_decompress_dense_tensor.argtypes = lib.excp_decompress_tensor.argtypes
    lib.excp_decompress_dense_checkpoint.argtypes = lib.excp_decompress_checkpoint.argtypes
    lib.excp_profile_enable.argtypes = [vp, C.c_int]
    lib.excp_set_kmeans_margin.argtypes = [vp, C.c_int]
    lib.excp_set_wait_limit.argtypes = [vp, C.c_ulonglong]
    lib.excp_set_report_sse.argtypes = [vp, C.c_int]
    lib.excp_selftest_wait_timeout.argtypes = [vp, C.c_ulonglong, vp]
    lib.excp_profile_stage_count.argtypes = []
    lib.excp_profile_stage_name.argtypes = [C.c_int]
    lib.excp_profile_stage_name.restype = C.c_char_p
    lib.excp_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_ulonglong)]
    lib.excp_mx4_bytes.argtypes = [sz, sz, C.c_int]
    lib.excp_mx4_bytes.restype = sz
    lib.excp_mx4_tensor_scale.argtypes = [vp, vp, C.c_int, sz, sz, sz, vp, vp]
    lib.excp_mx4_quantize.argtypes = [vp, vp, C.c_int, sz, sz, sz, C.c_int, vp, vp, vp]
    lib.excp_mx4_dequantize.argtypes = [vp, vp, sz, sz, C.c_int, vp, vp, C.c_int, sz, vp]
    lib.excp_mx4_matmul.argtypes = [vp, vp, sz, vp, vp, sz, vp, sz, C.c_int, vp, vp, C.c_int, sz, vp]
    lib.excp_mx4_linear_scratch.argtypes = [vp, sz, sz, sz, C.c_int]
    lib.excp_mx4_linear_scratch.restype = sz
    lib.excp_mx4_linear.argtypes = [vp, vp, C.c_int, sz, sz, vp, vp, sz, vp, sz, C.c_int, vp, vp, C.c_int, sz, vp, vp]
    lib.excp_token_logprobs.argtypes = [vp, vp, C.c_int, sz, sz, sz, vp, C.c_float, C.c_int, vp, vp, vp, vp, vp, vp]
    lib.excp_token_logprobs_grad.argtypes = [vp, vp, C.c_int, sz, sz, sz, vp, C.c_float, vp, vp, vp, vp, sz, vp]
    lib.excp_score_status.argtypes = [vp, vp]
    mat = C.POINTER(CMatrix)
    lib.excp_act8_bytes.argtypes = [sz, sz]
    lib.excp_act8_bytes.restype = sz
    lib.excp_act8_quantize.argtypes = [vp, mat, vp, vp]
    lib.excp_act8_restore.argtypes = [vp, vp, mat, vp]
    lib.excp_act_grad_scratch.argtypes = [vp, sz, sz]
    lib.excp_act_grad_scratch.restype = sz
    lib.excp_act_grad.argtypes = [vp, C.c_int, mat, mat, mat, mat, vp, vp, vp]
    lib.excp_layer_norm.argtypes = [vp, mat, vp, vp, C.c_int, C.c_float, C.c_int, mat, vp, vp, vp]
    lib.excp_layer_norm_grad_scratch.argtypes = [vp, sz, sz]
    lib.excp_layer_norm_grad_scratch.restype = sz
    lib.excp_layer_norm_grad.argtypes = [vp, mat, mat, vp, C.c_int, C.c_int, vp, mat, mat, vp, vp, vp, vp]
    lib.excp_linear_scratch.argtypes = [mat, mat]
    lib.excp_linear_scratch.restype = sz
    lib.excp_linear.argtypes = [vp, mat, mat, vp, C.c_int, C.c_int, mat, mat, mat, vp, vp]
    lib.excp_linear_grad_input.argtypes = [vp, mat, mat, mat, mat, vp, vp]
    lib.excp_linear_grad_weight.argtypes = [vp, mat, mat, mat, mat, vp, vp]
    for name in EXPORTS:
        if getattr(lib, name).restype is C.c_int:
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def load_scoring():
    """Loads (compiling it first if need be) the native half of the binding, which the scoring calls go through.  The first of them
    does so by itself; what compresses and restores needs neither it nor a host compiler."""
    global _score
    if isinstance(_score, _NotLoaded):
        lib = load_library()
        spec = importlib.util.spec_from_file_location(__package__ + "._score", _build.build_binding())
        native = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(native)
        native.bind(*[C.cast(getattr(lib, name), C.c_void_p).value for name in _SCORE_CALLS], ExcpError)
        _score = native
    return _score


def _ptr(t: torch.Tensor | None) -> int:
    return 0 if t is None or t.numel() == 0 else t.data_ptr()


def _check_f32_cuda(*ts: torch.Tensor) -> None:
    for t in ts:
        if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            raise TypeError("expected contiguous float32 CUDA tensors")


WEIGHTS_F32, WEIGHTS_F16, WEIGHTS_BF16 = 0, 1, 2
_WEIGHT_DTYPE = {WEIGHTS_F32: torch.float32, WEIGHTS_F16: torch.float16, WEIGHTS_BF16: torch.bfloat16}


def _check_weights(weight_format: int, *ts: torch.Tensor) -> None:
    for t in ts:
        if not (t.is_cuda and t.dtype == _WEIGHT_DTYPE[weight_format] and t.is_contiguous()):
            raise TypeError(f"expected contiguous {_WEIGHT_DTYPE[weight_format]} CUDA tensors")


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def record_bytes(numel: int, nnz_w: int, nnz_o: int, bits: int = 4) -> int:
    return load_library().excp_record_bytes(numel, nnz_w, nnz_o, bits)


def dense_bytes(numel: int, bits: int = 4) -> int:
    return load_library().excp_dense_bytes(numel, bits)


def compress_bound(numel: int, bits: int = 4) -> int:
    return load_library().excp_compress_bound(numel, bits)


NOALLOC_MAX_NUMEL = 1 << 24


def decompress_tensor_noalloc(blob: torch.Tensor, blob_bytes: int, w_prev, w_out, ea_out, eas_out) -> None:
    """excp_decompress_tensor_noalloc: decode one record on the current device without a handle
    and without any allocation by the library (for restore paths that cannot allocate: the
    device is fully reserved by the framework's allocator, or cudaMalloc's device-wide
    synchronisation is not acceptable).  Tensors of more than NOALLOC_MAX_NUMEL elements are
    refused; calls must not overlap on the GPU."""
    _check_f32_cuda(w_prev, w_out, ea_out, eas_out)
    st = load_library().excp_decompress_tensor_noalloc(blob.data_ptr(), blob_bytes, _ptr(w_prev), w_prev.numel(),
                                                       _ptr(w_out), _ptr(ea_out), _ptr(eas_out), _stream())
    if st != 0:
        raise ExcpError(st, "excp_decompress_tensor_noalloc")


# ---- scoring a restored checkpoint ---------------------------------------------
MX4_FORMAT = {"e8m0_32": 1, "e4m3_16": 2}
_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def mx4_bytes(rows: int, cols: int, fmt: str) -> int:
    """Size of a packed 4-bit matrix (layout: include/excp.h)."""
    return load_library().excp_mx4_bytes(rows, cols, MX4_FORMAT[fmt])


class Mx4Matrix:
    """A packed 4-bit matrix: `data` (uint8, mx4_bytes), its shape, its format ("e8m0_32" or "e4m3_16") and, for
    the latter, the tensor scale (a float32 tensor of one value on the same device; None = 1)."""
    __slots__ = ("data", "rows", "cols", "fmt", "scale", "code")

    def __init__(self, data: torch.Tensor, rows: int, cols: int, fmt: str, scale: torch.Tensor | None = None):
        self.data, self.rows, self.cols, self.fmt, self.scale = data, rows, cols, fmt, scale
        self.code = MX4_FORMAT[fmt]


class TokenLogprobs:
    """What token_logprobs returns: logprob and entropy (float32 [rows]), top_logprob (float32) and top_index (int64,
    [rows, top]; None without alternatives), row_stats (float32 [rows, 4]) and scale for the gradient.  logprob and entropy
    share their memory, top_logprob and top_index share theirs, and of a few rows (512 bytes in all) everything does: a clone
    takes one out."""
    __slots__ = ("logprob", "entropy", "top_logprob", "top_index", "row_stats", "scale")

    def __init__(self, logprob, entropy, top_logprob, top_index, row_stats, scale):
        self.logprob, self.entropy, self.top_logprob, self.top_index = logprob, entropy, top_logprob, top_index
        self.row_stats, self.scale = row_stats, scale


# ---- the layers before the logits, and the way back -------------------------------
ACTIVATIONS = {"none": 0, "gelu": 1, "gelu_tanh": 2, "silu": 3}


def act8_bytes(rows: int, cols: int) -> int:
    """Size of a packed 8-bit matrix (layout: include/excp.h)."""
    return load_library().excp_act8_bytes(rows, cols)


class Act8Matrix:
    """Values kept in 8 bits: `data` (uint8, act8_bytes) and the shape."""
    __slots__ = ("data", "rows", "cols")

    def __init__(self, data: torch.Tensor, rows: int, cols: int):
        self.data, self.rows, self.cols = data, rows, cols


class Norm:
    """What layer_norm returns: y, row_stats (float32 [rows, 2]: mean and 1 / deviation), kept (x as an Act8Matrix, or None) and rms."""
    __slots__ = ("y", "row_stats", "kept", "rms")

    def __init__(self, y, row_stats, kept, rms):
        self.y, self.row_stats, self.kept, self.rms = y, row_stats, kept, rms


class NormGrad:
    """What layer_norm_grad returns: dx, and dweight and dbias (float32; None where not wanted, dbias also for rms)."""
    __slots__ = ("dx", "dweight", "dbias")

    def __init__(self, dx, dweight, dbias):
        self.dx, self.dweight, self.dbias = dx, dweight, dbias


class ActGrad:
    """What act_grad returns: dpre, a (the activation's value; None where not wanted) and dbias (float32)."""
    __slots__ = ("dpre", "a", "dbias")

    def __init__(self, dpre, a, dbias):
        self.dpre, self.a, self.dbias = dpre, a, dbias


def _kept(m):
    """The tensor of a plain or packed matrix, and whether it is packed."""
    return (m.data, True) if isinstance(m, Act8Matrix) else (m, False)


def _same_shape(m, like: torch.Tensor, what: str) -> None:
    if isinstance(m, Act8Matrix) and (m.rows, m.cols) != tuple(like.shape):
        raise TypeError(f"{what}: expected the shape {list(like.shape)}")


class Handle:
    """Owns the library's scratch workspace on one device (excp_create / excp_destroy).

    Calls on one handle share that workspace: they must be ordered on the device, on one stream or with events between
    streams (two tensor scales at once on two streams can both come out wrong).  Programs that score on several streams at
    once keep a handle for each."""

    def __init__(self, workspace_numel: int, device: int | None = None):
        self.lib = load_library()
        self.device = torch.cuda.current_device() if device is None else device
        self._h = C.c_void_p()
        st = self.lib.excp_create(C.byref(self._h), self.device, workspace_numel)
        if st != 0:
            raise ExcpError(st, "excp_create")

    def close(self) -> None:
        if self._h:
            self.lib.excp_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_cuda_error(self) -> int:
        e = C.c_int(0)
        self.lib.excp_last_cuda_error(self._h, C.byref(e))
        return e.value

    def set_kmeans_margin(self, margin: int) -> None:
        """excp_set_kmeans_margin: a tuning knob; the centres do not depend on it."""
        st = self.lib.excp_set_kmeans_margin(self._h, int(margin))
        if st != 0:
            raise ExcpError(st, "excp_set_kmeans_margin")

    def set_report_sse(self, on: bool = True) -> None:
        """excp_set_report_sse: fill sse_w, sse_ea, sse_eas of the statistics (off by default)."""
        st = self.lib.excp_set_report_sse(self._h, int(on))
        if st != 0:
            raise ExcpError(st, "excp_set_report_sse")

    def set_wait_limit(self, nanoseconds: int) -> None:
        """excp_set_wait_limit: how long a warp waits for an asynchronous copy before the call gives up."""
        st = self.lib.excp_set_wait_limit(self._h, int(nanoseconds))
        if st != 0:
            raise ExcpError(st, "excp_set_wait_limit")

    def selftest_wait_timeout(self, nanoseconds: int) -> int:
        """excp_selftest_wait_timeout: returns the status (EXCP_ERR_TIMEOUT = -7 is the expected one)."""
        return self.lib.excp_selftest_wait_timeout(self._h, int(nanoseconds), _stream())

    def profile_enable(self, on: bool = True) -> None:
        st = self.lib.excp_profile_enable(self._h, int(on))
        if st != 0:
            raise ExcpError(st, "excp_profile_enable")

    def profile_read(self):
        """(dict stage name -> ms of the last call, kernel launches of the last call)."""
        n = self.lib.excp_profile_stage_count()
        ms = (C.c_double * n)()
        launches = C.c_ulonglong(0)
        self.lib.excp_profile_read(self._h, ms, C.byref(launches))
        return {self.lib.excp_profile_stage_name(i).decode(): ms[i] for i in range(n)}, launches.value

    # ---- Algorithm 1 -----------------------------------------------------
    def compress_tensor(self, p: Params, w_t, w_prev, ea, eas, blob_out: torch.Tensor):
        """excp_compress_tensor.  Returns (record bytes, stats)."""
        _check_f32_cuda(w_t, w_prev, ea, eas)
        cp, nbytes, stats = p.to_c(), C.c_size_t(0), CStats()
        st = self.lib.excp_compress_tensor(self._h, C.byref(cp), _ptr(w_t), _ptr(w_prev), _ptr(ea), _ptr(eas),
                                           w_t.numel(), blob_out.data_ptr(), blob_out.numel() * blob_out.element_size(),
                                           C.byref(nbytes), C.byref(stats), _stream())
        if st != 0:
            raise ExcpError(st, "excp_compress_tensor")
        return nbytes.value, stats

    def compress_checkpoint(self, p: Params, tensors, blob_out: torch.Tensor, want_stats: bool = True,
                            weight_format: int = WEIGHTS_F32, tensor_indices=None):
        """excp_compress_checkpoint (or, for 16-bit weights, excp_compress_checkpoint_w16) over a list of
        (w_t, w_prev, ea, eas).  Returns (offsets list of len n+1, list of stats or None).  With
        `tensor_indices` (the tensors' places in the whole checkpoint, for a rank that compresses a share of
        it) the call is excp_compress_checkpoint_indexed."""
        n = len(tensors)
        for q in tensors:
            _check_weights(weight_format, q[0], q[1])
            _check_f32_cuda(q[2], q[3])
        arr = lambda k: (C.c_void_p * n)(*[_ptr(q[k]) for q in tensors])
        numel = (C.c_size_t * n)(*[q[0].numel() for q in tensors])
        offs = (C.c_size_t * (n + 1))()
        stats = (CStats * n)() if want_stats else None
        cp = p.to_c()
        cap = blob_out.numel() * blob_out.element_size()
        if tensor_indices is not None:
            if weight_format != WEIGHTS_F32 or len(tensor_indices) != n:
                raise ValueError("tensor_indices: one per tensor, fp32 weights only")
            idx = (C.c_size_t * n)(*[int(i) for i in tensor_indices])
            st = self.lib.excp_compress_checkpoint_indexed(self._h, C.byref(cp), n, arr(0), arr(1), arr(2), arr(3), numel, idx,
                                                           blob_out.data_ptr(), cap, offs, stats, _stream())
        elif weight_format == WEIGHTS_F32:
            st = self.lib.excp_compress_checkpoint(self._h, C.byref(cp), n, arr(0), arr(1), arr(2), arr(3), numel,
                                                   blob_out.data_ptr(), cap, offs, stats, _stream())
        else:
            st = self.lib.excp_compress_checkpoint_w16(self._h, C.byref(cp), n, arr(0), arr(1), arr(2), arr(3), numel,
                                                       weight_format, blob_out.data_ptr(), cap, offs, stats, _stream())
        if st != 0:
            raise ExcpError(st, "excp_compress_checkpoint" + ("" if weight_format == WEIGHTS_F32 else "_w16"))
        return list(offs), (list(stats) if want_stats else None)

    def compress_checkpoint_host(self, p: Params, tensors, blob_out: torch.Tensor, want_stats: bool = True):
        """excp_compress_checkpoint_host: `tensors` and `blob_out` are HOST tensors
        (page-locked for the copies to overlap the kernels)."""
        n = len(tensors)
        for q in tensors:
            for t in q:
                if t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous():
                    raise TypeError("expected contiguous float32 host tensors")
        if blob_out.is_cuda:
            raise TypeError("blob_out must be a host tensor")
        arr = lambda k: (C.c_void_p * n)(*[_ptr(q[k]) for q in tensors])
        numel = (C.c_size_t * n)(*[q[0].numel() for q in tensors])
        offs = (C.c_size_t * (n + 1))()
        stats = (CStats * n)() if want_stats else None
        cp = p.to_c()
        st = self.lib.excp_compress_checkpoint_host(self._h, C.byref(cp), n, arr(0), arr(1), arr(2), arr(3), numel,
                                                    blob_out.data_ptr(), blob_out.numel() * blob_out.element_size(),
                                                    offs, stats, _stream())
        if st != 0:
            raise ExcpError(st, "excp_compress_checkpoint_host")
        return list(offs), (list(stats) if want_stats else None)

    # ---- Algorithm 2 -----------------------------------------------------
    def decompress_tensor(self, blob: torch.Tensor, blob_bytes: int, w_prev, w_out, ea_out, eas_out) -> None:
        _check_f32_cuda(w_prev, w_out, ea_out, eas_out)
        st = self.lib.excp_decompress_tensor(self._h, blob.data_ptr(), blob_bytes, _ptr(w_prev), w_prev.numel(),
                                             _ptr(w_out), _ptr(ea_out), _ptr(eas_out), _stream())
        if st != 0:
            raise ExcpError(st, "excp_decompress_tensor")

    def decompress_checkpoint(self, blob: torch.Tensor, offsets, w_prev, w_out, ea_out, eas_out,
                              dense: bool = False, weight_format: int = WEIGHTS_F32) -> None:
        n = len(w_prev)
        _check_weights(weight_format, *w_prev, *w_out)
        _check_f32_cuda(*ea_out, *eas_out)
        arr = lambda ts: (C.c_void_p * n)(*[_ptr(t) for t in ts])
        numel = (C.c_size_t * n)(*[t.numel() for t in w_prev])
        offs = (C.c_size_t * (n + 1))(*offsets)
        if weight_format != WEIGHTS_F32:
            if dense:
                raise ValueError("the dense layout decodes to fp32 weights only")
            st = self.lib.excp_decompress_checkpoint_w16(self._h, blob.data_ptr(), offs, n, arr(w_prev), numel,
                                                         weight_format, arr(w_out), arr(ea_out), arr(eas_out), _stream())
            if st != 0:
                raise ExcpError(st, "excp_decompress_checkpoint_w16")
            return
        fn = self.lib.excp_decompress_dense_checkpoint if dense else self.lib.excp_decompress_checkpoint
        st = fn(self._h, blob.data_ptr(), offs, n, arr(w_prev), numel, arr(w_out), arr(ea_out), arr(eas_out),
                _stream())
        if st != 0:
            raise ExcpError(st, "excp_decompress_dense_checkpoint" if dense else "excp_decompress_checkpoint")

    # ---- the dense index layout (Sections 3.3 / 4.2) ----------------------
    def record_to_dense(self, record: torch.Tensor, record_bytes: int, numel: int, dense_out: torch.Tensor) -> int:
        out = C.c_size_t(0)
        st = self.lib.excp_record_to_dense(self._h, record.data_ptr(), record_bytes, numel, dense_out.data_ptr(),
                                           dense_out.numel(), C.byref(out), _stream())
        if st != 0:
            raise ExcpError(st, "excp_record_to_dense")
        return out.value

    def checkpoint_to_dense(self, blob: torch.Tensor, offsets, numels, dense_out: torch.Tensor) -> list[int]:
        n = len(numels)
        offs = (C.c_size_t * (n + 1))(*offsets)
        numel = (C.c_size_t * n)(*numels)
        douts = (C.c_size_t * (n + 1))()
        st = self.lib.excp_checkpoint_to_dense(self._h, blob.data_ptr(), offs, n, numel, dense_out.data_ptr(),
                                               dense_out.numel(), douts, _stream())
        if st != 0:
            raise ExcpError(st, "excp_checkpoint_to_dense")
        return list(douts)

    def decompress_dense_tensor(self, dense: torch.Tensor, dense_bytes_: int, w_prev, w_out, ea_out, eas_out) -> None:
        _check_f32_cuda(w_prev, w_out, ea_out, eas_out)
        st = self.lib.excp_decompress_dense_tensor(self._h, dense.data_ptr(), dense_bytes_, _ptr(w_prev),
                                                   w_prev.numel(), _ptr(w_out), _ptr(ea_out), _ptr(eas_out), _stream())
        if st != 0:
            raise ExcpError(st, "excp_decompress_dense_tensor")

    # ---- scoring a restored checkpoint -------------------------------------
    # Only enqueued on the current stream; results are allocated by torch where the caller gives no `out`.  The arguments
    # are marshalled by csrc/score_binding.cpp: TypeError for tensors of the wrong kind, ExcpError for a status.
    # torch's autograd sees none of these calls: results carry no graph, also of inputs that require a gradient.  The
    # gradient of the log probabilities is token_logprobs_grad; through a packed matrix there is none.
    def mx4_tensor_scale(self, x: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        """excp_mx4_tensor_scale: the tensor scale of a matrix, as a float32 tensor of one value."""
        return _score.mx4_tensor_scale(self._h.value, self.device, x, out)

    def mx4_quantize(self, x: torch.Tensor, fmt: str, tensor_scale: torch.Tensor | None = None,
                     out: torch.Tensor | None = None) -> Mx4Matrix:
        """excp_mx4_quantize: x [rows, cols] as a packed 4-bit matrix (into `out`, uint8, if given)."""
        data = _score.mx4_quantize(self._h.value, self.device, x, MX4_FORMAT[fmt], tensor_scale, out)
        rows, cols = x.shape
        return Mx4Matrix(data, rows, cols, fmt, tensor_scale)

    def mx4_dequantize(self, m: Mx4Matrix, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
        """excp_mx4_dequantize: the values that the codes stand for."""
        return _score.mx4_dequantize(self._h.value, self.device, m.data, m.rows, m.cols, m.code, m.scale, dtype, out)

    def mx4_matmul(self, a: Mx4Matrix, b: Mx4Matrix, bias: torch.Tensor | None = None, dtype: torch.dtype = torch.bfloat16,
                   out: torch.Tensor | None = None) -> torch.Tensor:
        """excp_mx4_matmul: a b^T (+ bias per row of b) of two packed matrices, [a.rows, b.rows]."""
        if a.code != b.code or a.cols != b.cols:
            raise TypeError("a, b: expected the same format and number of columns")
        return _score.mx4_matmul(self._h.value, self.device, a.data, a.rows, a.scale, b.data, b.rows, b.scale, a.cols, a.code, bias,
                                 dtype, out)

    def mx4_linear(self, x: torch.Tensor, w: Mx4Matrix, bias: torch.Tensor | None = None, tensor_scale: torch.Tensor | None = None,
                   out: torch.Tensor | None = None, dtype: torch.dtype | None = None, x_packed: torch.Tensor | None = None) -> torch.Tensor:
        """excp_mx4_linear: x w^T (+ bias), x [rows, w.cols] quantised to w's format with the tensor scale given; the result
        has x's type unless `dtype` or `out` says otherwise.  `x_packed` (uint8, excp_mx4_linear_scratch bytes) is room for
        the packed x."""
        return _score.mx4_linear(self._h.value, self.device, x, tensor_scale, w.data, w.rows, w.scale, w.cols, w.code, bias, dtype, out,
                                 x_packed)

    def token_logprobs(self, logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, scale: float = 1.0) -> TokenLogprobs:
        """excp_token_logprobs: log probability of each row's token, entropy, and the `top` likeliest alternatives."""
        return TokenLogprobs(*_score.token_logprobs(self._h.value, self.device, logits, tokens, top, scale), scale)

    def token_logprobs_grad(self, logits: torch.Tensor, tokens: torch.Tensor, r: TokenLogprobs, g_logprob: torch.Tensor | None,
                            g_entropy: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        """excp_token_logprobs_grad: the gradient with respect to the logits, from what token_logprobs returned for them.
        `out` may be `logits`."""
        return _score.token_logprobs_grad(self._h.value, self.device, logits, tokens, r.row_stats, r.scale, g_logprob, g_entropy, out)

    # ---- the layers before the logits, and the way back ----------------------
    # As the scoring calls: only enqueued, and marshalled natively.  Autograd records none of them: results carry no graph, also of inputs that
    # require a gradient (what is written into an `out` moves its version).  The gradients are calls of their own.
    def act8_quantize(self, x: torch.Tensor, out: torch.Tensor | None = None) -> Act8Matrix:
        """excp_act8_quantize: x [rows, cols] in 8 bits (into `out`, uint8, if given).  Not recorded by autograd."""
        data = _score.act8_quantize(self._h.value, self.device, x, out)
        rows, cols = x.shape
        return Act8Matrix(data, rows, cols)

    def act8_restore(self, m: Act8Matrix, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
        """excp_act8_restore: the values that the codes stand for.  Not recorded by autograd."""
        return _score.act8_restore(self._h.value, self.device, m.data, m.rows, m.cols, dtype, out)

    def act_grad(self, dy: torch.Tensor, pre: torch.Tensor | Act8Matrix, act: str, again: bool = False, bias: bool = True,
                 out: torch.Tensor | None = None) -> ActGrad:
        """excp_act_grad: the gradient through an activation ("gelu", "gelu_tanh", "silu") from what went into it (`pre`, plain or in 8 bits),
        the bias's gradient, and with `again` the activation's value.  `out` (for dpre) may be dy.  Not recorded by autograd."""
        _same_shape(pre, dy, "pre")
        data, is_packed = _kept(pre)
        return ActGrad(*_score.act_grad(self._h.value, self.device, dy, data, is_packed, ACTIVATIONS[act], True, again, bias, out))

    def bias_grad(self, dy: torch.Tensor) -> torch.Tensor:
        """excp_act_grad without an activation: the sum of dy's rows, float32.  Not recorded by autograd."""
        return _score.act_grad(self._h.value, self.device, dy, None, False, 0, False, False, True, None)[2]

    def layer_norm(self, x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5, rms: bool = False,
                   keep: bool = False, out: torch.Tensor | None = None) -> Norm:
        """excp_layer_norm: the norm of every row of x (rms: without mean and bias); with `keep` also x in 8 bits.  `out` may be x.
        Not recorded by autograd: the gradient is layer_norm_grad."""
        y, stats, data = _score.layer_norm(self._h.value, self.device, x, weight, bias, eps, rms, keep, out)
        return Norm(y, stats, None if data is None else Act8Matrix(data, *x.shape), rms)

    def layer_norm_grad(self, dy: torch.Tensor, x: torch.Tensor | Act8Matrix, weight: torch.Tensor | None, r: Norm, add: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, vectors: bool = True) -> NormGrad:
        """excp_layer_norm_grad: the gradients of x (plus `add`), weight and bias, from what layer_norm returned for them; x may be r.kept.
        `out` (for dx) may be dy or add.  Not recorded by autograd."""
        _same_shape(x, dy, "x")
        data, is_packed = _kept(x)
        return NormGrad(*_score.layer_norm_grad(self._h.value, self.device, dy, data, is_packed, weight, r.rms, r.row_stats, add, out, vectors))

    def linear(self, x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, act: str = "none", residual: torch.Tensor | None = None,
               out: torch.Tensor | None = None, dtype: torch.dtype | None = None) -> torch.Tensor:
        """excp_linear: act(x w^T + bias) + residual of 16-bit matrices; the result has x's type unless `dtype` or `out` says otherwise.
        `out` may be the residual.  Not recorded by autograd: the gradients are linear_grad_input, linear_grad_weight, act_grad and bias_grad."""
        return _score.linear(self._h.value, self.device, x, w, bias, ACTIVATIONS[act], residual, dtype, out, None)[0]

    def linear_kept(self, x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, act: str = "none", residual: torch.Tensor | None = None,
                    keep: str | torch.dtype = "act8", out: torch.Tensor | None = None, dtype: torch.dtype | None = None):
        """The same, and what goes into the activation: an Act8Matrix for keep="act8", else a tensor of that type.  With many rows the result may
        round to the other neighbour than linear's where float32 is kept, or "act8" without an activation (excp.h: sums)."""
        if isinstance(keep, str) and keep != "act8":
            raise ValueError('keep: "act8" or a torch.dtype')
        y, data = _score.linear(self._h.value, self.device, x, w, bias, ACTIVATIONS[act], residual, dtype, out, True if keep == "act8" else keep)
        return y, Act8Matrix(data, x.shape[0], w.shape[0]) if keep == "act8" else data

    def linear_grad_input(self, dy: torch.Tensor, w: torch.Tensor, add: torch.Tensor | None = None, out: torch.Tensor | None = None,
                          dtype: torch.dtype | None = None) -> torch.Tensor:
        """excp_linear_grad_input: dy w (+ add), in dy's type unless `dtype` or `out` says otherwise.  `out` may be add.  Not
        recorded by autograd."""
        return _score.linear_grad_input(self._h.value, self.device, dy, w, add, dtype, out)

    def linear_grad_weight(self, dy: torch.Tensor, x: torch.Tensor, add: torch.Tensor | None = None, out: torch.Tensor | None = None,
                           dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """excp_linear_grad_weight: dy^T x (+ add).  `out` may be add (gradients summed over several calls).  Not recorded by autograd."""
        return _score.linear_grad_weight(self._h.value, self.device, dy, x, add, dtype, out)

    def score_status(self) -> None:
        """excp_score_status: synchronises; raises if a product's bounded wait ran out since the last report."""
        st = self.lib.excp_score_status(self._h, torch.cuda.current_stream(self.device).cuda_stream)
        if st != 0:
            raise ExcpError(st, "excp_score_status")
