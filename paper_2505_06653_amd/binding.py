"""Thin ctypes binding of include/bof4.h: argument marshalling only, every step of the path runs in the HIP library.

torch supplies device memory (tensors) and the stream; nothing is computed here.  The functions carry the names of
the C entry points.  A missing library is an error (there is no fallback of any kind).

`stream` of a call is the torch.cuda.Stream that it enqueues on (default: the current one).  What the call allocates belongs to
that stream; the caller sees to it that its own tensors are ready there and that they live until the call is done with them.
The calls know nothing of autograd: what they return carries no graph, whatever their inputs require.  A
torch.autograd.Function joins a call and its gradient (its backward gets the tensors that the forward call wrote: pre, stats,
entropy).
"""
import ctypes
import os
import struct

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbof4_hip.so")

BOF4_OK, BOF4_ERR_ARG, BOF4_ERR_CAPACITY, BOF4_ERR_WORKSPACE, BOF4_ERR_HIP = 0, -1, -2, -3, -4
EXPORTS = ("bof4_workspace_bytes", "bof4_opq_threshold", "bof4_thresholds", "bof4_bin_table", "bof4_lloyd_step",
           "bof4_codebook_update", "bof4_lloyd_step_mae", "bof4_codebook_update_mae", "bof4_quantize",
           "bof4_dequantize", "bof4_quantize_begin", "bof4_quantize_finish", "bof4_lloyd_step_begin", "bof4_wait_result",
           "bof4_lloyd_step_static", "bof4_quantize_lloyd", "bof4_quantize_lloyd_begin", "bof4_quantize_lloyd_finish",
           "bof4_quant_error", "bof4_gemv", "bof4_gemv_outlier_table",
           "bof4_gemv_outlier_table_bytes", "bof4_gemm", "bof4_gemm_pack", "bof4_gemm_packed_bytes",
           "bof4_gemm_outlier_table", "bof4_gemm_workspace_bytes",
           "bof4_gemv_linear", "bof4_gemm_linear", "bof4_gemm_linear_workspace_bytes", "bof4_gemm_linear_backward",
           "bof4_gemm_linear_backward_workspace_bytes", "bof4_token_logprobs", "bof4_token_logprobs_workspace_bytes",
           "bof4_token_logprobs_backward",
           "bof4_theory_centroids", "bof4_theory_workspace_bytes", "bof4_time_next_call", "bof4_last_error",
           "bof4_last_hip_error")


class Bof4Error(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"bof4 error {code}: {msg}")
        self.code = code


class LloydStats(ctypes.Structure):
    _fields_ = [("num", ctypes.c_double * 16), ("den", ctypes.c_double * 16), ("cnt", ctypes.c_uint64 * 16),
                ("sse", ctypes.c_double), ("n_used", ctypes.c_uint64), ("n_outliers", ctypes.c_uint64)]

    def as_dict(self):
        return {"num": np.array(self.num[:], dtype=np.float64), "den": np.array(self.den[:], dtype=np.float64),
                "cnt": np.array(self.cnt[:], dtype=np.uint64), "sse": float(self.sse),
                "n_used": int(self.n_used), "n_outliers": int(self.n_outliers)}


class ErrorStats(ctypes.Structure):
    _fields_ = [("sse", ctypes.c_double), ("sae", ctypes.c_double), ("max_abs", ctypes.c_double),
                ("n_outliers", ctypes.c_uint64), ("n", ctypes.c_uint64)]

    def as_dict(self):
        return {"sse": self.sse, "sae": self.sae, "max_abs": self.max_abs, "n_outliers": int(self.n_outliers),
                "n": int(self.n)}


class MaeStats(ctypes.Structure):
    _fields_ = [("median", ctypes.c_double * 16), ("den", ctypes.c_double * 16), ("cnt", ctypes.c_uint64 * 16),
                ("sae", ctypes.c_double), ("n_used", ctypes.c_uint64), ("n_outliers", ctypes.c_uint64)]

    def as_dict(self):
        return {"median": np.array(self.median[:], dtype=np.float64), "den": np.array(self.den[:], dtype=np.float64),
                "cnt": np.array(self.cnt[:], dtype=np.uint64), "sae": float(self.sae),
                "n_used": int(self.n_used), "n_outliers": int(self.n_outliers)}


# bof4_layer and bof4_layer_gradient of include/bof4.h, packed: act and five types, five or six addresses, row strides
LAYER = struct.Struct("@6I5P4Q")
LAYER_GRADIENT = struct.Struct("@6I6P5Q")


_lib = None


def lib():
    """Load libbof4_hip.so (built by `python -m paper_2505_06653_amd.build`); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not built - run `python -m paper_2505_06653_amd.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, f64p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_double)
        L.bof4_workspace_bytes.restype = ctypes.c_size_t
        L.bof4_workspace_bytes.argtypes = [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint64]
        L.bof4_opq_threshold.restype = ctypes.c_double
        L.bof4_opq_threshold.argtypes = [ctypes.c_double, ctypes.c_uint32]
        L.bof4_thresholds.restype = ctypes.c_int
        L.bof4_thresholds.argtypes = [f64p, ctypes.POINTER(ctypes.c_float)]
        L.bof4_bin_table.restype = ctypes.c_int
        L.bof4_bin_table.argtypes = [f64p, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_uint32),
                                     ctypes.POINTER(ctypes.c_int)]
        L.bof4_lloyd_step.restype = ctypes.c_int
        L.bof4_lloyd_step.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                      ctypes.c_int, ctypes.POINTER(LloydStats), vp, ctypes.c_size_t, vp]
        L.bof4_codebook_update.restype = ctypes.c_int
        L.bof4_codebook_update.argtypes = [ctypes.POINTER(LloydStats), ctypes.c_uint16, vp]
        L.bof4_lloyd_step_mae.restype = ctypes.c_int
        L.bof4_lloyd_step_mae.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                          ctypes.c_int, ctypes.c_uint16, ctypes.POINTER(MaeStats), vp, ctypes.c_size_t,
                                          vp]
        L.bof4_codebook_update_mae.restype = ctypes.c_int
        L.bof4_codebook_update_mae.argtypes = [ctypes.POINTER(MaeStats), ctypes.c_uint16, vp]
        L.bof4_quantize.restype = ctypes.c_int
        L.bof4_quantize.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                    vp, vp, vp, vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64), vp,
                                    ctypes.c_size_t, vp]
        for name in ("bof4_quantize_begin", "bof4_quantize_finish"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = L.bof4_quantize.argtypes
        for name in ("bof4_quantize_lloyd", "bof4_quantize_lloyd_begin", "bof4_quantize_lloyd_finish"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                         ctypes.c_int, vp, vp, vp, vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64),
                                         ctypes.POINTER(LloydStats), vp, ctypes.c_size_t, vp]
        L.bof4_lloyd_step_begin.restype = ctypes.c_int
        L.bof4_lloyd_step_begin.argtypes = L.bof4_lloyd_step.argtypes
        L.bof4_lloyd_step_static.restype = ctypes.c_int
        L.bof4_lloyd_step_static.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                             ctypes.c_int, ctypes.POINTER(LloydStats), vp]
        L.bof4_wait_result.restype = ctypes.c_int
        L.bof4_wait_result.argtypes = [vp, vp]
        L.bof4_dequantize.restype = ctypes.c_int
        L.bof4_dequantize.argtypes = [vp, vp, ctypes.c_uint64, ctypes.c_uint32, f64p, vp, vp, ctypes.c_uint64, vp, vp]
        L.bof4_quant_error.restype = ctypes.c_int
        L.bof4_quant_error.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, f64p, ctypes.c_int, ctypes.c_double,
                                       ctypes.POINTER(ErrorStats), vp, ctypes.c_size_t, vp]
        L.bof4_gemv.restype = ctypes.c_int
        L.bof4_gemv.argtypes = [vp, vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, f64p, vp, ctypes.c_uint64,
                                vp, ctypes.c_uint32, vp, vp]
        L.bof4_gemv_outlier_table.restype = ctypes.c_int
        L.bof4_gemv_outlier_table.argtypes = [vp, vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, f64p, vp, vp,
                                              ctypes.c_uint64, vp, ctypes.c_size_t, vp]
        L.bof4_gemv_outlier_table_bytes.restype = ctypes.c_size_t
        L.bof4_gemv_outlier_table_bytes.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint64]
        L.bof4_gemm.restype = ctypes.c_int
        L.bof4_gemm.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint64, f64p, vp, ctypes.c_uint64, vp, ctypes.c_uint32,
                                vp, vp, ctypes.c_size_t, vp]
        L.bof4_gemm_pack.restype = ctypes.c_int
        L.bof4_gemm_pack.argtypes = [vp, vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, vp, ctypes.c_size_t, vp]
        L.bof4_gemm_packed_bytes.restype = ctypes.c_size_t
        L.bof4_gemm_packed_bytes.argtypes = [ctypes.c_uint64, ctypes.c_uint64]
        L.bof4_gemm_outlier_table.restype = ctypes.c_int
        L.bof4_gemm_outlier_table.argtypes = L.bof4_gemv_outlier_table.argtypes
        L.bof4_gemm_workspace_bytes.restype = ctypes.c_size_t
        L.bof4_gemm_workspace_bytes.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32]
        u32, u64, size = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t
        L.bof4_gemv_linear.restype = ctypes.c_int
        L.bof4_gemv_linear.argtypes = [vp, vp, u64, u64, u32, f64p, vp, u64, vp, u32, vp, vp]
        L.bof4_gemm_linear.restype = ctypes.c_int
        L.bof4_gemm_linear.argtypes = [vp, u64, u64, f64p, vp, u64, vp, u32, vp, vp, size, vp]
        L.bof4_gemm_linear_backward.restype = ctypes.c_int
        L.bof4_gemm_linear_backward.argtypes = [vp, u64, u64, f64p, vp, u64, u32, vp, vp, size, vp]
        for name in ("bof4_gemm_linear_workspace_bytes", "bof4_gemm_linear_backward_workspace_bytes"):
            getattr(L, name).restype = size
            getattr(L, name).argtypes = [u64, u64, u32]
        L.bof4_token_logprobs.restype = ctypes.c_int
        L.bof4_token_logprobs.argtypes = [vp, u32, u64, u64, u64, vp, u32, vp, vp, vp, vp, vp, vp, size, vp]
        L.bof4_token_logprobs_workspace_bytes.restype = size
        L.bof4_token_logprobs_workspace_bytes.argtypes = [u64, u64, u32]
        L.bof4_token_logprobs_backward.restype = ctypes.c_int
        L.bof4_token_logprobs_backward.argtypes = [vp, u32, u64, u64, u64, vp, vp, vp, vp, vp, vp, u32, u64, vp]
        L.bof4_theory_workspace_bytes.restype = ctypes.c_size_t
        L.bof4_theory_workspace_bytes.argtypes = [ctypes.c_uint32]
        L.bof4_theory_centroids.restype = ctypes.c_int
        L.bof4_theory_centroids.argtypes = [f64p, f64p, ctypes.c_uint32, ctypes.c_double, ctypes.c_uint32, f64p,
                                            ctypes.c_uint16, ctypes.c_int, f64p, vp, ctypes.c_size_t, vp]
        L.bof4_time_next_call.restype = ctypes.c_int
        L.bof4_time_next_call.argtypes = [vp, vp]
        L.bof4_last_error.restype = ctypes.c_char_p
        L.bof4_last_hip_error.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(code, allow=()):
    if code != BOF4_OK and code not in allow:
        raise Bof4Error(code, lib().bof4_last_error().decode())
    return code


_F64P = ctypes.POINTER(ctypes.c_double)
_cb_cache = {}  # id(array) -> (array, pointer); holding the array keeps its id from being reused


def _cb(cb):
    """Codebook as a contiguous float64[16] array plus its ctypes pointer.  Arrays that already have that form are
    passed through, and their pointer object is kept (building one costs more than the rest of a call's marshalling)."""
    hit = _cb_cache.get(id(cb))
    if hit is not None and hit[0] is cb:
        return cb, hit[1]
    arr = cb if (type(cb) is np.ndarray and cb.dtype == np.float64 and cb.flags.c_contiguous) \
        else np.ascontiguousarray(cb, dtype=np.float64)
    if arr.shape != (16,):
        raise ValueError("codebook must have 16 levels")
    ptr = arr.ctypes.data_as(_F64P)
    if arr is cb:
        if len(_cb_cache) >= 16:
            _cb_cache.clear()
        _cb_cache[id(cb)] = (cb, ptr)
    return arr, ptr


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


try:
    _raw_stream = torch._C._cuda_getCurrentRawStream  # the current stream's handle without building a Stream object
except AttributeError:  # pragma: no cover
    _raw_stream = None


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if _raw_stream is not None:
        return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _empty(shape, dtype, device, stream):
    """A tensor for a call on `stream` (None: the current one), out of that stream's memory: it is not what another stream still
    works on, and once it is dropped it goes to nobody who does not wait for the call."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _result(shape, dtype, device, stream):
    """The same for a result: the caller works with it on the current stream as well, which has to be done with it, too, before
    the memory of a dropped one is used again."""
    t = _empty(shape, dtype, device, stream)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream())
    return t


def bof4_workspace_bytes(n, block, out_capacity=0):
    return int(lib().bof4_workspace_bytes(n, block, out_capacity))


def bof4_opq_threshold(q, block):
    return float(lib().bof4_opq_threshold(q, block))


def bof4_thresholds(cb):
    cb, cbp = _cb(cb)
    thr = np.zeros(15, dtype=np.float32)
    _check(lib().bof4_thresholds(cbp, thr.ctypes.data_as(ctypes.POINTER(ctypes.c_float))))
    return thr


def bof4_bin_table(cb):
    """Returns (thr float32[33], base uint32[33], fast bool)."""
    cb, cbp = _cb(cb)
    thr = np.zeros(33, dtype=np.float32)
    base = np.zeros(33, dtype=np.uint32)
    fast = ctypes.c_int(0)
    _check(lib().bof4_bin_table(cbp, thr.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                base.ctypes.data_as(ctypes.POINTER(ctypes.c_uint32)), ctypes.byref(fast)))
    return thr, base, bool(fast.value)


def bof4_codebook_update(stats, pinned_mask, cb):
    """stats: LloydStats (as returned by bof4_lloyd_step(..., raw=True)) or its dict form.  Returns new float64[16]."""
    out = np.array(cb, dtype=np.float64)  # a copy: the C function updates in place
    if out.shape != (16,):
        raise ValueError("codebook must have 16 levels")
    if not isinstance(stats, LloydStats):
        s = LloydStats()
        for l in range(16):
            s.num[l], s.den[l], s.cnt[l] = float(stats["num"][l]), float(stats["den"][l]), int(stats["cnt"][l])
        s.sse, s.n_used, s.n_outliers = float(stats["sse"]), int(stats["n_used"]), int(stats["n_outliers"])
        stats = s
    _check(lib().bof4_codebook_update(ctypes.byref(stats), pinned_mask, out.ctypes.data))
    return out


def bof4_theory_centroids(pdf, cdf, u_max, block, cb, pinned_mask, signed, ws=None, stream=None, device="cuda"):
    """One theoretical maximisation step for the distribution tabulated in pdf / cdf (float64 arrays over [0, u_max]).
    Returns the new float64[16] codebook."""
    pdf = np.ascontiguousarray(pdf, dtype=np.float64)
    cdf = np.ascontiguousarray(cdf, dtype=np.float64)
    if pdf.shape != cdf.shape or pdf.ndim != 1:
        raise ValueError("pdf and cdf must be 1-d arrays of one length")
    cb, cbp = _cb(cb)
    n = int(pdf.size)
    if ws is None:
        ws = _empty(int(lib().bof4_theory_workspace_bytes(n)), torch.uint8, device, stream)
    out = np.zeros(16, dtype=np.float64)
    _check(lib().bof4_theory_centroids(pdf.ctypes.data_as(_F64P), cdf.ctypes.data_as(_F64P), n, float(u_max), block,
                                       cbp, int(pinned_mask), int(signed), out.ctypes.data_as(_F64P), _ptr(ws),
                                       ws.numel(), _stream(stream)))
    return out


def bof4_time_next_call(start_event, stop_event):
    """start_event / stop_event: torch.cuda.Event(enable_timing=True) that have been recorded once (so that their
    HIP handles exist); the next call records them around its main kernel."""
    _check(lib().bof4_time_next_call(ctypes.c_void_p(start_event.cuda_event), ctypes.c_void_p(stop_event.cuda_event)))


def alloc_workspace(n, block, out_capacity=0, device="cuda", stream=None):
    """A workspace for calls on `stream` (default: the current one)."""
    nbytes = max(bof4_workspace_bytes(n, block, out_capacity), 256)
    return _empty(nbytes, torch.uint8, device, stream)


def pinned_lloyd_stats():
    """A LloydStats record in pinned host memory (the GPU then writes results in place).  Returns (struct, keepalive)."""
    buf = torch.zeros(ctypes.sizeof(LloydStats), dtype=torch.uint8).pin_memory()
    return LloydStats.from_address(buf.data_ptr()), buf


def pinned_mae_stats():
    """A MaeStats record in pinned host memory.  Returns (struct, keepalive)."""
    buf = torch.zeros(ctypes.sizeof(MaeStats), dtype=torch.uint8).pin_memory()
    return MaeStats.from_address(buf.data_ptr()), buf


def pinned_counter():
    """A uint64 outlier counter in pinned host memory.  Returns (ctypes.c_uint64, keepalive)."""
    buf = torch.zeros(1, dtype=torch.int64).pin_memory()
    return ctypes.c_uint64.from_address(buf.data_ptr()), buf


def pinned_error_stats():
    """An ErrorStats record in pinned host memory.  Returns (struct, keepalive)."""
    buf = torch.zeros(ctypes.sizeof(ErrorStats), dtype=torch.uint8).pin_memory()
    return ErrorStats.from_address(buf.data_ptr()), buf


def bof4_quant_error(w, block, cb, signed, opq_T=0.0, ws=None, stream=None, out=None):
    """Quantisation error of the flat bf16 device tensor w: dict with sse, sae, max_abs, n_outliers, n."""
    cb, cbp = _cb(cb)
    n = w.numel()
    if ws is None:
        ws = alloc_workspace(n, block, 0, w.device, stream)
    rec = out if out is not None else ErrorStats()
    _check(lib().bof4_quant_error(_ptr(w), n, block, cbp, int(signed), float(opq_T), ctypes.byref(rec), _ptr(ws),
                                  ws.numel(), _stream(stream)))
    return rec.as_dict()


def bof4_gemv_outlier_table_bytes(rows, cols, n_outliers):
    return int(lib().bof4_gemv_outlier_table_bytes(rows, cols, n_outliers))


def bof4_gemv_outlier_table(codes, scales, rows, cols, block, cb, out_idx, out_val, n_outliers=None, out=None,
                            stream=None):
    """The outlier list of one quantised matrix in the form bof4_gemv reads (uint8 device tensor; made once)."""
    cb, cbp = _cb(cb)
    k = 0 if out_idx is None else int(out_idx.numel())
    if n_outliers is not None:
        if n_outliers > k:
            raise ValueError("n_outliers exceeds the list")
        k = int(n_outliers)
    if out is None:
        out = _result(bof4_gemv_outlier_table_bytes(rows, cols, k), torch.uint8, codes.device, stream)
    _check(lib().bof4_gemv_outlier_table(_ptr(codes), _ptr(scales), rows, cols, block, cbp,
                                         _ptr(out_idx) if k else None, _ptr(out_val) if k else None, k, _ptr(out),
                                         out.numel(), _stream(stream)))
    return out


def _tokens(x, cols):
    """x as [n_tokens, cols]; one token may come as [cols]."""
    x2 = x[None, :] if x.dim() == 1 else x
    if x2.dim() != 2 or x2.dtype != torch.bfloat16 or x2.shape[1] != cols or not x2.is_contiguous():
        raise ValueError("x must be a contiguous bfloat16 tensor of [n_tokens, cols]")
    return x2


def bof4_gemv(codes, scales, rows, cols, block, cb, x, table=None, n_outliers=0, out=None, stream=None):
    """y = x W~^T for the quantised row-major [rows, cols] matrix; x is bf16 [n_tokens, cols] (or [cols]) on the
    device, the result float32 [n_tokens, rows].  `table` (bof4_gemv_outlier_table) brings n_outliers outliers in."""
    cb, cbp = _cb(cb)
    x2 = _tokens(x, cols)
    n_tokens = int(x2.shape[0])
    if out is None:
        out = _result((n_tokens, rows), torch.float32, x.device, stream)
    k = int(n_outliers)
    if k and table is None:
        raise ValueError("outliers need their table (bof4_gemv_outlier_table)")
    _check(lib().bof4_gemv(_ptr(codes), _ptr(scales), rows, cols, block, cbp, _ptr(table) if k else None, k,
                           _ptr(x2), n_tokens, _ptr(out), _stream(stream)))
    return out


def bof4_gemm_workspace_bytes(rows, cols, n_tokens):
    return int(lib().bof4_gemm_workspace_bytes(rows, cols, n_tokens))


def bof4_gemm_outlier_table(codes, scales, rows, cols, block, cb, out_idx, out_val, n_outliers=None, out=None,
                            stream=None):
    """The outlier list of one quantised matrix in the form bof4_gemm reads (uint8 device tensor; made once)."""
    cb, cbp = _cb(cb)
    k = 0 if out_idx is None else int(out_idx.numel())
    if n_outliers is not None:
        if n_outliers > k:
            raise ValueError("n_outliers exceeds the list")
        k = int(n_outliers)
    if out is None:
        out = _result(bof4_gemv_outlier_table_bytes(rows, cols, k), torch.uint8, codes.device, stream)
    _check(lib().bof4_gemm_outlier_table(_ptr(codes), _ptr(scales), rows, cols, block, cbp,
                                         _ptr(out_idx) if k else None, _ptr(out_val) if k else None, k, _ptr(out),
                                         out.numel(), _stream(stream)))
    return out


def bof4_gemm_packed_bytes(rows, cols):
    return int(lib().bof4_gemm_packed_bytes(rows, cols))


def bof4_gemm_pack(codes, scales, rows, cols, block, out=None, stream=None):
    """Codes and block constants of one quantised matrix in the order bof4_gemm reads them (uint8 device tensor;
    made once)."""
    if out is None:
        out = _result(bof4_gemm_packed_bytes(rows, cols), torch.uint8, codes.device, stream)
    _check(lib().bof4_gemm_pack(_ptr(codes), _ptr(scales), rows, cols, block, _ptr(out), out.numel(), _stream(stream)))
    return out


def bof4_gemm(packed, rows, cols, cb, x, table=None, n_outliers=0, out=None, ws=None, stream=None):
    """y = x W^^T for the decoded (bfloat16) form of the quantised row-major [rows, cols] matrix, given as
    bof4_gemm_pack made it; x is bf16 [n_tokens, cols] on the device, the result float32 [n_tokens, rows].  `table`
    (bof4_gemm_outlier_table) brings n_outliers outliers in; `ws`: optional uint8 device tensor of
    bof4_gemm_workspace_bytes(...) bytes."""
    cb, cbp = _cb(cb)
    x2 = _tokens(x, cols)
    if packed.numel() < bof4_gemm_packed_bytes(rows, cols):
        raise ValueError("packed matrix too small for rows x cols (bof4_gemm_pack)")
    n_tokens = int(x2.shape[0])
    if out is None:
        out = _result((n_tokens, rows), torch.float32, x.device, stream)
    k = int(n_outliers)
    if k and table is None:
        raise ValueError("outliers need their table (bof4_gemm_outlier_table)")
    if ws is None:
        ws = _empty(bof4_gemm_workspace_bytes(rows, cols, n_tokens), torch.uint8, x.device, stream)
    _check(lib().bof4_gemm(_ptr(packed), rows, cols, cbp, _ptr(table) if k else None, k, _ptr(x2), n_tokens,
                           _ptr(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out


def bof4_lloyd_step(w, block, cb, signed, opq_T=0.0, weight_by_max2=True, ws=None, stream=None, raw=False, out=None):
    """w: flat bf16 device tensor.  Returns the statistics as a dict (or the ctypes struct with raw=True).
    `out`: optional LloydStats to fill (e.g. from pinned_lloyd_stats())."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    n = w.numel()
    cb, cbp = _cb(cb)
    if ws is None:
        ws = alloc_workspace(n, block, 0, w.device, stream)
    if out is None:
        out = LloydStats()
    _check(lib().bof4_lloyd_step(_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max2)),
                                 ctypes.byref(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out if raw else out.as_dict()


def bof4_lloyd_step_mae(w, block, cb, signed, opq_T=0.0, skip_mask=0, ws=None, stream=None, raw=False, out=None,
                        weight_by_max=True):
    """MAE criterion: per-region weighted medians (weight_by_max=False: plain medians of the normalised weights).
    w: flat bf16 device tensor.  skip_mask: regions (pinned levels) whose median is not wanted.  Returns the statistics as a dict (or the ctypes struct with raw=True)."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    n = w.numel()
    cb, cbp = _cb(cb)
    if ws is None:
        ws = alloc_workspace(n, block, 0, w.device, stream)
    if out is None:
        out = MaeStats()
    _check(lib().bof4_lloyd_step_mae(_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max)),
                                     int(skip_mask),
                                     ctypes.byref(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out if raw else out.as_dict()


def bof4_codebook_update_mae(stats, pinned_mask, cb):
    """stats: MaeStats or its dict form.  Returns new float64[16]."""
    out = np.array(cb, dtype=np.float64)
    if out.shape != (16,):
        raise ValueError("codebook must have 16 levels")
    if not isinstance(stats, MaeStats):
        s = MaeStats()
        for l in range(16):
            s.median[l], s.den[l], s.cnt[l] = float(stats["median"][l]), float(stats["den"][l]), int(stats["cnt"][l])
        s.sae, s.n_used, s.n_outliers = float(stats["sae"]), int(stats["n_used"]), int(stats["n_outliers"])
        stats = s
    _check(lib().bof4_codebook_update_mae(ctypes.byref(stats), pinned_mask, out.ctypes.data))
    return out


def bof4_quantize(w, block, cb, signed, opq_T=0.0, out_capacity=0, codes=None, scales=None, out_idx=None,
                  out_val=None, ws=None, stream=None, allow_overflow=False, counter=None, trim=True):
    """w: flat bf16 device tensor.  Returns (codes u8[n/2], scales f16[n/block], out_idx i64[k], out_val f16[k],
    n_outliers).  Output tensors are allocated here unless passed in; trim=False returns the outlier buffers whole
    (the first n_outliers entries are the list)."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    n = w.numel()
    dev = w.device
    cb, cbp = _cb(cb)
    if codes is None:
        codes = _result(max(n // 2, 1), torch.uint8, dev, stream)
    if scales is None:
        scales = _result(max(n // max(block, 1), 1), torch.float16, dev, stream)
    if opq_T > 0:
        if out_idx is None:
            out_idx = _result(max(out_capacity, 1), torch.int64, dev, stream)
        if out_val is None:
            out_val = _result(max(out_capacity, 1), torch.float16, dev, stream)
        if ws is None:
            ws = alloc_workspace(n, block, out_capacity, dev, stream)
    nout = counter if counter is not None else ctypes.c_uint64(0)
    code = lib().bof4_quantize(_ptr(w), n, block, cbp, int(signed), float(opq_T), _ptr(codes), _ptr(scales),
                               _ptr(out_idx), _ptr(out_val), out_capacity, ctypes.byref(nout), _ptr(ws),
                               0 if ws is None else ws.numel(), _stream(stream))
    _check(code, allow=(BOF4_ERR_CAPACITY,) if allow_overflow else ())
    if not trim:
        return codes, scales, out_idx, out_val, int(nout.value)
    k = min(int(nout.value), out_capacity)
    return (codes, scales, None if out_idx is None else out_idx[:k], None if out_val is None else out_val[:k],
            int(nout.value))


def bof4_quantize_lloyd(w, block, cb, signed, opq_T=0.0, out_capacity=0, weight_by_max2=True, codes=None, scales=None,
                        out_idx=None, out_val=None, ws=None, stream=None, allow_overflow=False, counter=None,
                        stats=None, trim=True, raw=False):
    """bof4_quantize and bof4_lloyd_step in one pass.  Returns (codes, scales, out_idx, out_val, n_outliers, stats):
    the first five as bof4_quantize returns them, stats as bof4_lloyd_step does (dict, or the struct with raw=True)."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    n = w.numel()
    dev = w.device
    cb, cbp = _cb(cb)
    if codes is None:
        codes = _result(max(n // 2, 1), torch.uint8, dev, stream)
    if scales is None:
        scales = _result(max(n // max(block, 1), 1), torch.float16, dev, stream)
    if opq_T > 0:
        if out_idx is None:
            out_idx = _result(max(out_capacity, 1), torch.int64, dev, stream)
        if out_val is None:
            out_val = _result(max(out_capacity, 1), torch.float16, dev, stream)
    if ws is None:
        ws = alloc_workspace(n, block, out_capacity, dev, stream)
    nout = counter if counter is not None else ctypes.c_uint64(0)
    st = stats if stats is not None else LloydStats()
    code = lib().bof4_quantize_lloyd(_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max2)),
                                     _ptr(codes), _ptr(scales), _ptr(out_idx), _ptr(out_val), out_capacity,
                                     ctypes.byref(nout), ctypes.byref(st), _ptr(ws), ws.numel(), _stream(stream))
    _check(code, allow=(BOF4_ERR_CAPACITY,) if allow_overflow else ())
    stats_out = st if raw else st.as_dict()
    if not trim:
        return codes, scales, out_idx, out_val, int(nout.value), stats_out
    k = min(int(nout.value), out_capacity)
    return (codes, scales, None if out_idx is None else out_idx[:k], None if out_val is None else out_val[:k],
            int(nout.value), stats_out)


class QuantizeLloydInFlight:
    """bof4_quantize_lloyd_begin has been called with these arguments; finish() waits for the outlier count and
    returns it (the sums: bof4_wait_result(stats))."""

    def __init__(self, args, counter, keep):
        self.args, self.counter, self.keep = args, counter, keep

    def finish(self, allow_overflow=False):
        code = lib().bof4_quantize_lloyd_finish(*self.args)
        _check(code, allow=(BOF4_ERR_CAPACITY,) if allow_overflow else ())
        return int(self.counter.value)


def bof4_quantize_lloyd_begin(w, block, cb, signed, opq_T, out_capacity, codes, scales, out_idx, out_val, ws, counter,
                              stats, weight_by_max2=True, stream=None):
    """Enqueues bof4_quantize_lloyd into caller-owned buffers (counter: pinned_counter(), stats:
    pinned_lloyd_stats()) and returns a QuantizeLloydInFlight."""
    n = w.numel()
    cb, cbp = _cb(cb)
    args = (_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max2)), _ptr(codes), _ptr(scales),
            _ptr(out_idx), _ptr(out_val), out_capacity, ctypes.byref(counter), ctypes.byref(stats), _ptr(ws),
            0 if ws is None else ws.numel(), _stream(stream))
    _check(lib().bof4_quantize_lloyd_begin(*args))
    return QuantizeLloydInFlight(args, counter, (w, cb, codes, scales, out_idx, out_val, ws, stats))


class QuantizeInFlight:
    """bof4_quantize_begin has been called with these arguments; finish() waits for the outlier count and returns it."""

    def __init__(self, args, counter, keep):
        self.args, self.counter, self.keep = args, counter, keep

    def finish(self, allow_overflow=False):
        code = lib().bof4_quantize_finish(*self.args)
        _check(code, allow=(BOF4_ERR_CAPACITY,) if allow_overflow else ())
        return int(self.counter.value)


def bof4_quantize_begin(w, block, cb, signed, opq_T, out_capacity, codes, scales, out_idx, out_val, ws, counter,
                        stream=None):
    """Enqueues bof4_quantize into caller-owned buffers (counter: from pinned_counter()) and returns a
    QuantizeInFlight; other work may be enqueued on the stream before its finish() is called."""
    n = w.numel()
    cb, cbp = _cb(cb)
    args = (_ptr(w), n, block, cbp, int(signed), float(opq_T), _ptr(codes), _ptr(scales), _ptr(out_idx),
            _ptr(out_val), out_capacity, ctypes.byref(counter), _ptr(ws), 0 if ws is None else ws.numel(),
            _stream(stream))
    _check(lib().bof4_quantize_begin(*args))
    return QuantizeInFlight(args, counter, (w, cb, codes, scales, out_idx, out_val, ws))


def bof4_lloyd_step_begin(w, block, cb, signed, out, opq_T=0.0, weight_by_max2=True, ws=None, stream=None):
    """Enqueues bof4_lloyd_step; `out` is a LloydStats in pinned host memory (pinned_lloyd_stats()), complete after
    bof4_wait_result(out)."""
    n = w.numel()
    cb, cbp = _cb(cb)
    if ws is None:
        ws = alloc_workspace(n, block, 0, w.device, stream)
    _check(lib().bof4_lloyd_step_begin(_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max2)),
                                       ctypes.byref(out), _ptr(ws), ws.numel(), _stream(stream)))
    return out


def bof4_lloyd_step_static(w, block, cb, signed, out, opq_T=0.0, weight_by_max2=True, stream=None, n=None):
    """bof4_lloyd_step without a workspace argument (the library's own fixed device array holds the partial sums; no
    allocation anywhere in the call).  `out`: a LloydStats in pinned host memory (pinned_lloyd_stats()).  `n`: number
    of weights, if not all of w."""
    n = w.numel() if n is None else int(n)
    cb, cbp = _cb(cb)
    _check(lib().bof4_lloyd_step_static(_ptr(w), n, block, cbp, int(signed), float(opq_T), int(bool(weight_by_max2)),
                                        ctypes.byref(out), _stream(stream)))
    return out


def bof4_wait_result(stats, stream=None):
    """Waits until the GPU has written the record `stats` (LloydStats / MaeStats: word n_used; ErrorStats: word n)."""
    field = "n" if isinstance(stats, ErrorStats) else "n_used"
    addr = ctypes.addressof(stats) + getattr(type(stats), field).offset
    _check(lib().bof4_wait_result(ctypes.c_void_p(addr), _stream(stream)))
    return stats


def bof4_dequantize(codes, scales, n, block, cb, out_idx=None, out_val=None, out=None, stream=None, n_outliers=None):
    """Returns the flat bf16 device tensor of n dequantised weights.  The outlier list is the first n_outliers
    entries of out_idx / out_val (all of them if n_outliers is None)."""
    cb, cbp = _cb(cb)
    if out is None:
        out = _result(n, torch.bfloat16, codes.device, stream)
    k = 0 if out_idx is None else int(out_idx.numel())
    if n_outliers is not None:
        if n_outliers > k:
            raise ValueError("n_outliers exceeds the list")
        k = int(n_outliers)
    _check(lib().bof4_dequantize(_ptr(codes), _ptr(scales), n, block, cbp, _ptr(out_idx) if k else None,
                                 _ptr(out_val) if k else None, k, _ptr(out), _stream(stream)))
    return out


_TYPES = {torch.float32: 0, torch.bfloat16: 1}  # BOF4_F32, BOF4_BF16


def _tensor(t, name, dtypes, shape, dev):
    """The address of a tensor of one of `dtypes` and of that shape (None: any), its last dimension contiguous, on the current
    device `dev` (the library enqueues on that)."""
    if t.get_device() != dev or t.dtype not in dtypes or (shape is not None and t.shape != shape) or \
            (not t.is_contiguous() and t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be of {' or '.join(str(d) for d in dtypes)}, of the shape {shape or tuple(t.shape)}, on the "
                         f"current GPU and contiguous in its last dimension: got {t.dtype}, {tuple(t.shape)}, {t.device}, strides "
                         f"{t.stride()}")
    return t.data_ptr()


def _row_stride(t):
    """Elements from one row of a 2-d tensor to the next (a single row's stride says nothing)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _flat(t, name, dtypes, shape, dev):
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return _tensor(t, name, dtypes, shape, dev)


_F32, _I64, _U8 = (torch.float32,), (torch.int64,), (torch.uint8,)


def _scratch(ws, nbytes, device, stream, gpu):
    """The caller's workspace, or one of `nbytes`."""
    if ws is not None:
        _flat(ws, "ws", _U8, None, gpu)
        return ws
    return _empty(max(int(nbytes), 1), torch.uint8, device, stream)


def _gpu(stream):
    """The current device, on which the tensors of a call and its stream have to be."""
    gpu = torch.cuda.current_device()
    if stream is not None and stream.device_index != gpu:
        raise ValueError(f"stream must be one of the current GPU: got one of device {stream.device_index}")
    return gpu


ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}  # BOF4_ACT_*


def _activation(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _layer_input(x, cols, gpu):
    x2 = _tokens(x, cols)
    if x2.get_device() != gpu:
        raise ValueError("x must be on the current GPU")
    return x2


def _table(table, rows, cols, n_outliers, gpu):
    """The address of an outlier table for that matrix and list, or None without a list."""
    k = int(n_outliers)
    if k == 0:
        return None, 0
    if table is None:
        raise ValueError("outliers need their table (bof4_gemv_outlier_table, bof4_gemm_outlier_table)")
    # (bof4_gemv_outlier_table_bytes)
    if table.get_device() != gpu or not table.is_contiguous() or table.numel() < (((rows * -(-cols // 2048) + 1) * 4 + 7) & ~7) + 8 * k:
        raise ValueError("the outlier table must be on the current GPU, contiguous, of bof4_gemv_outlier_table_bytes(rows, cols, n_outliers) bytes")
    return table.data_ptr(), k


def _packed(packed, rows, cols, gpu):
    if packed.get_device() != gpu or not packed.is_contiguous() or packed.numel() < bof4_gemm_packed_bytes(rows, cols):
        raise ValueError("the packed matrix must be on the current GPU, contiguous and not too small for rows x cols (bof4_gemm_pack)")
    return packed.data_ptr()


def _layer(n_tokens, rows, bias, act, mul, residual, pre, out, gpu):
    shape = (n_tokens, rows)
    bias_at = mul_at = residual_at = pre_at = bias_type = mul_type = residual_type = pre_type = ld_mul = ld_residual = ld_pre = 0
    if bias is not None:
        bias_at, bias_type = _flat(bias, "bias", _TYPES, (rows,), gpu), _TYPES[bias.dtype]
    if mul is not None:
        mul_at, mul_type, ld_mul = _tensor(mul, "mul", _TYPES, shape, gpu), _TYPES[mul.dtype], _row_stride(mul)
    if residual is not None:
        residual_at, residual_type = _tensor(residual, "residual", _TYPES, shape, gpu), _TYPES[residual.dtype]
        ld_residual = _row_stride(residual)
    if pre is not None:
        pre_at, pre_type, ld_pre = _tensor(pre, "pre", _TYPES, shape, gpu), _TYPES[pre.dtype], _row_stride(pre)
    out_at = _tensor(out, "out", _TYPES, shape, gpu)
    return LAYER.pack(_activation(act), bias_type, mul_type, residual_type, _TYPES[out.dtype], pre_type, bias_at, mul_at,
                      residual_at, out_at, pre_at, ld_mul, ld_residual, _row_stride(out), ld_pre)


def bof4_gemv_linear(codes, scales, rows, cols, block, cb, x, table=None, n_outliers=0, bias=None, act="none", mul=None,
                     residual=None, pre=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """y = act(x W~^T + bias) * mul + residual for one token to a few; matrix, x, table as for bof4_gemv.  bias [rows], mul,
    residual, pre, out [n_tokens, rows] (rows of any stride): bfloat16 or float32 each.  act: a key of ACTIVATIONS.  `pre`: a
    tensor that receives x W~^T + bias; `out`: the result's, may be mul or the residual (else of `out_dtype`)."""
    cb, cbp = _cb(cb)
    gpu = _gpu(stream)
    x2 = _layer_input(x, cols, gpu)
    n_tokens = x2.shape[0]
    table_at, k = _table(table, rows, cols, n_outliers, gpu)
    if codes.get_device() != gpu or scales.get_device() != gpu or 2 * codes.numel() < rows * cols or scales.numel() * block < rows * cols \
            or not codes.is_contiguous() or not scales.is_contiguous() or scales.element_size() != 2:
        raise ValueError("codes and scales (2 bytes each) must be on the current GPU, contiguous, and those of rows x cols weights")
    if out is None:
        out = _result((n_tokens, rows), out_dtype, x.device, stream)
    layer = _layer(n_tokens, rows, bias, act, mul, residual, pre, out, gpu)
    _check(lib().bof4_gemv_linear(codes.data_ptr(), scales.data_ptr(), rows, cols, block, cbp, table_at, k, x2.data_ptr(),
                                  n_tokens, layer, _stream(stream)))
    return out


def bof4_gemm_linear_workspace_bytes(rows, cols, n_tokens):
    return int(lib().bof4_gemm_linear_workspace_bytes(rows, cols, n_tokens))


def bof4_gemm_linear(packed, rows, cols, cb, x, table=None, n_outliers=0, bias=None, act="none", mul=None, residual=None,
                     pre=None, out=None, out_dtype=torch.bfloat16, ws=None, stream=None):
    """y = act(x W^^T + bias) * mul + residual for many tokens; matrix, x, table as for bof4_gemm, the rest as for
    bof4_gemv_linear; `ws`: optional uint8 device tensor of bof4_gemm_linear_workspace_bytes(...) bytes."""
    cb, cbp = _cb(cb)
    gpu = _gpu(stream)
    x2 = _layer_input(x, cols, gpu)
    packed_at = _packed(packed, rows, cols, gpu)
    n_tokens = x2.shape[0]
    table_at, k = _table(table, rows, cols, n_outliers, gpu)
    if out is None:
        out = _result((n_tokens, rows), out_dtype, x.device, stream)
    layer = _layer(n_tokens, rows, bias, act, mul, residual, pre, out, gpu)
    ws = _scratch(ws, 0 if ws is not None else bof4_gemm_linear_workspace_bytes(rows, cols, n_tokens), x.device, stream, gpu)
    _check(lib().bof4_gemm_linear(packed_at, rows, cols, cbp, table_at, k, x2.data_ptr(), n_tokens, layer, ws.data_ptr(),
                                  ws.numel(), _stream(stream)))
    return out


def bof4_gemm_linear_backward_workspace_bytes(rows, cols, n_tokens):
    return int(lib().bof4_gemm_linear_backward_workspace_bytes(rows, cols, n_tokens))


def bof4_gemm_linear_backward(packed, rows, cols, cb, dy, table=None, n_outliers=0, act="none", pre=None, mul=None, dmul=None,
                              dbias=None, out=None, out_dtype=torch.bfloat16, ws=None, stream=None):
    """The gradients of bof4_gemm_linear: returns dx [n_tokens, cols] (`out`, else of `out_dtype`) from dy [n_tokens, rows] and,
    as the forward call had them, act, pre (what it wrote) and mul.  `dmul` [n_tokens, rows] and `dbias` float32 [rows]: tensors
    that receive those gradients (the residual's is dy).  dy * mul * act'(pre) enters the product rounded to bfloat16 if dy and dx
    are bfloat16, in sixteen bits if dy is float32, whole if dx is float32 (two and three times the products)."""
    cb, cbp = _cb(cb)
    if dy.dim() != 2 or dy.shape[1] != rows:
        raise ValueError("dy must be [n_tokens, rows]")
    gpu, n_tokens = _gpu(stream), dy.shape[0]
    packed_at = _packed(packed, rows, cols, gpu)
    table_at, k = _table(table, rows, cols, n_outliers, gpu)
    if out is None:
        out = _result((n_tokens, cols), out_dtype, dy.device, stream)
    shape = (n_tokens, rows)
    pre_at = mul_at = dmul_at = dbias_at = pre_type = mul_type = dmul_type = ld_pre = ld_mul = ld_dmul = 0
    dy_at, dx_at = _tensor(dy, "dy", _TYPES, shape, gpu), _tensor(out, "out", _TYPES, (n_tokens, cols), gpu)
    if pre is not None:
        pre_at, pre_type, ld_pre = _tensor(pre, "pre", _TYPES, shape, gpu), _TYPES[pre.dtype], _row_stride(pre)
    if mul is not None:
        mul_at, mul_type, ld_mul = _tensor(mul, "mul", _TYPES, shape, gpu), _TYPES[mul.dtype], _row_stride(mul)
    if dmul is not None:
        dmul_at, dmul_type, ld_dmul = _tensor(dmul, "dmul", _TYPES, shape, gpu), _TYPES[dmul.dtype], _row_stride(dmul)
    if dbias is not None:
        dbias_at = _flat(dbias, "dbias", _F32, (rows,), gpu)
    g = LAYER_GRADIENT.pack(_activation(act), _TYPES[dy.dtype], pre_type, mul_type, dmul_type, _TYPES[out.dtype], dy_at, pre_at,
                            mul_at, dmul_at, dbias_at, dx_at, _row_stride(dy), ld_pre, ld_mul, ld_dmul, _row_stride(out))
    ws = _scratch(ws, 0 if ws is not None else bof4_gemm_linear_backward_workspace_bytes(rows, cols, n_tokens), dy.device, stream, gpu)
    _check(lib().bof4_gemm_linear_backward(packed_at, rows, cols, cbp, table_at, k, n_tokens, g, ws.data_ptr(), ws.numel(),
                                           _stream(stream)))
    return out


def bof4_token_logprobs_workspace_bytes(n_rows, vocab, top=0):
    return int(lib().bof4_token_logprobs_workspace_bytes(n_rows, vocab, top))


def bof4_token_logprobs(logits, targets=None, top=0, ws=None, stream=None):
    """logits: float32 or bfloat16 [n_rows, vocab] on the device, rows of any stride; targets: int64 [n_rows] (below 0: no
    token asked for).  Returns (logprob float32 [n_rows] or None without targets, entropy float32 [n_rows], top_idx int64
    [n_rows, top] and top_logprob float32 [n_rows, top] or None with top = 0, stats float32 [n_rows, 2])."""
    gpu = _gpu(stream)
    logits_at = _tensor(logits, "logits", _TYPES, None, gpu)
    if logits.dim() != 2:
        raise ValueError("logits must be [n_rows, vocab]")
    n, vocab = logits.shape
    f32, top = torch.float32, int(top)
    new = logits.new_empty if stream is None else lambda shape, dtype: _result(shape, dtype, logits.device, stream)
    if top < 0:
        raise ValueError("top must not be negative")
    logprob = top_idx = top_logprob = targets_at = logprob_at = idx_at = top_at = None
    stats, entropy = new((n, 2), dtype=f32), new(n, dtype=f32)
    if targets is not None:
        targets_at, logprob = _flat(targets, "targets", _I64, (n,), gpu), new(n, dtype=f32)
        logprob_at = logprob.data_ptr()
    if top > 0:
        top_idx, top_logprob = new((n, top), dtype=torch.int64), new((n, top), dtype=f32)
        idx_at, top_at = top_idx.data_ptr(), top_logprob.data_ptr()
    ws = _scratch(ws, 0 if ws is not None else bof4_token_logprobs_workspace_bytes(n, vocab, top), logits.device, stream, gpu)
    _check(lib().bof4_token_logprobs(logits_at, _TYPES[logits.dtype], n, vocab, _row_stride(logits), targets_at, top,
                                     logprob_at, entropy.data_ptr(), idx_at, top_at, stats.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _stream(stream)))
    return logprob, entropy, top_idx, top_logprob, stats


def bof4_token_logprobs_backward(logits, stats, targets=None, d_logprob=None, entropy=None, d_entropy=None, out=None,
                                 out_dtype=None, stream=None):
    """The gradient by the logits, [n_rows, vocab], from bof4_token_logprobs' stats (and entropy) and the gradients of its
    logprob and entropy (float32 [n_rows]; None: that output is not used).  `out`: a tensor to fill, may be the logits."""
    gpu = _gpu(stream)
    logits_at = _tensor(logits, "logits", _TYPES, None, gpu)
    if logits.dim() != 2:
        raise ValueError("logits must be [n_rows, vocab]")
    n, vocab = logits.shape
    if (targets is None) != (d_logprob is None) or (entropy is None) != (d_entropy is None):
        raise ValueError("targets come with d_logprob, the entropy with d_entropy")
    targets_at = d_logprob_at = entropy_at = d_entropy_at = None
    if targets is not None:
        targets_at, d_logprob_at = _flat(targets, "targets", _I64, (n,), gpu), _flat(d_logprob, "d_logprob", _F32, (n,), gpu)
    if entropy is not None:
        entropy_at, d_entropy_at = _flat(entropy, "entropy", _F32, (n,), gpu), _flat(d_entropy, "d_entropy", _F32, (n,), gpu)
    if out is None:
        out = _result((n, vocab), out_dtype or logits.dtype, logits.device, stream)
    out_at = _tensor(out, "out", _TYPES, (n, vocab), gpu)
    _check(lib().bof4_token_logprobs_backward(logits_at, _TYPES[logits.dtype], n, vocab, _row_stride(logits),
                                              _flat(stats, "stats", _F32, (n, 2), gpu), targets_at, d_logprob_at, entropy_at,
                                              d_entropy_at, out_at, _TYPES[out.dtype], _row_stride(out), _stream(stream)))
    return out
