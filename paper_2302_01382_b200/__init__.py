"""Thin Python binding of the qcfg C-ABI library (include/qcfg.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch is used for device memory and streams.  The shared library is loaded on first
use; if it is missing and cannot be built the call fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

from .build import LIB, build_library

OK = 0
PER_TENSOR, PER_ROW = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU_TANH = 0, 1, 2
SEARCH_BISECTION, SEARCH_GREEDY = 0, 1
FORMS = ("conv_gather", "conv_im2col", "conv_slab", "conv_streamed", "shortcut", "rows", "narrow_fp32")
STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "EBITS", 3: "ESHAPE", 4: "EALIGN", 5: "ENOMEM", 6: "ENONFINITE", 7: "EARCH",
                8: "ECUDA", 9: "ETIMEOUT", 11: "ESTATE", 12: "EPAGE"}
EINVAL, EBITS, ESHAPE, EALIGN, ENOMEM, ENONFINITE, EARCH, ECUDA, ETIMEOUT = range(1, 10)
ESTATE, EPAGE = 11, 12
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

EXPORTS = ["qcfg_create", "qcfg_destroy", "qcfg_sync_status", "qcfg_selftest_wait_timeout", "qcfg_last_error", "qcfg_launch_count",
           "qcfg_set_fusion", "qcfg_set_pair_tiles", "qcfg_set_grouping", "qcfg_set_prefix_reuse", "qcfg_set_implicit_conv", "qcfg_set_gemm_chains", "qcfg_profile_enable", "qcfg_profile_read", "qcfg_calibrate", "qcfg_scales_from_absmax", "qcfg_quantize",
           "qcfg_quant_error_sweep", "qcfg_quant_error_sweep_static", "qcfg_gemm_i8", "qcfg_gemm_i8_requant", "qcfg_gemm_bf16",
           "qcfg_quantize_tokens", "qcfg_gemm_i8_token", "qcfg_linear_i8_work", "qcfg_linear_i8", "qcfg_kv_extend", "qcfg_kv_free", "qcfg_kv_fork",
           "qcfg_kv_compact", "qcfg_kv_copy_pages", "qcfg_kv_append", "qcfg_kv_read", "qcfg_kv_attention_work", "qcfg_kv_attention", "qcfg_model_create", "qcfg_model_set_attention",
           "qcfg_model_destroy", "qcfg_calibrate_model", "qcfg_model_act_absmax",
           "qcfg_model_weight_absmax", "qcfg_eval_config", "qcfg_latency_table", "qcfg_config_cost", "qcfg_noise_sensitivity", "qcfg_search", "qcfg_adjust_scales", "qcfg_scale_gradients", "qcfg_model_scales",
           "qcfg_model_reset_scales", "qcfg_debug_dump", "qcfg_debug_launch_forms"]


class QcfgError(RuntimeError):
    def __init__(self, status: int, msg: str = ""):
        name = STATUS_NAMES.get(status, str(status))
        super().__init__(f"QCFG_{name}: {msg}")
        self.status = status


class LayerStruct(C.Structure):
    _fields_ = [("w_dev", C.c_void_p), ("n_out", C.c_int64), ("k_in", C.c_int64), ("src", C.c_int32),
                ("src_col0", C.c_int32), ("act", C.c_int32), ("kh", C.c_int32), ("kw", C.c_int32),
                ("stride", C.c_int32), ("pad", C.c_int32), ("in_h", C.c_int32), ("in_w", C.c_int32),
                ("in_c", C.c_int32), ("pool_before", C.c_int32), ("src_h", C.c_int32), ("src_w", C.c_int32),
                ("residual_from", C.c_int32)]


class PoolStruct(C.Structure):
    _fields_ = [("table_dev", C.c_void_p), ("len_dev", C.c_void_p), ("refs_dev", C.c_void_p), ("n_pages", C.c_int32),
                ("page_tokens", C.c_int32), ("max_seqs", C.c_int32), ("max_pages", C.c_int32), ("refused_dev", C.c_void_p)]


class CacheStruct(C.Structure):
    _fields_ = [("k_dev", C.c_void_p), ("v_dev", C.c_void_p), ("k_absmax_dev", C.c_void_p), ("v_absmax_dev", C.c_void_p),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class BatchStruct(C.Structure):
    _fields_ = [("seqs_dev", C.c_void_p), ("starts_dev", C.c_void_p), ("n", C.c_int32), ("n_rows", C.c_int64)]


_lib = None


def load_library() -> C.CDLL:
    """Loads libqcfg.so (building it with nvcc first if it is absent)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB):
        build_library()
    lib = C.CDLL(LIB)
    vp, i64, i32, ci, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_int, C.c_float
    pool, cache, batch = C.POINTER(PoolStruct), C.POINTER(CacheStruct), C.POINTER(BatchStruct)
    sig = {
        "qcfg_create": [C.POINTER(vp), ci],
        "qcfg_destroy": [vp],
        "qcfg_sync_status": [vp, vp],
        "qcfg_selftest_wait_timeout": [vp, C.c_uint64, vp],
        "qcfg_set_fusion": [vp, ci],
        "qcfg_set_pair_tiles": [vp, ci],
        "qcfg_set_grouping": [vp, ci],
        "qcfg_set_prefix_reuse": [vp, ci],
        "qcfg_set_implicit_conv": [vp, ci],
        "qcfg_set_gemm_chains": [vp, ci],
        "qcfg_profile_enable": [vp, ci],
        "qcfg_profile_read": [vp, ci, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(C.c_double), ci],
        "qcfg_calibrate": [vp, vp, i64, i64, i64, ci, vp, vp],
        "qcfg_scales_from_absmax": [vp, vp, i64, ci, vp, vp, vp],
        "qcfg_quantize": [vp, vp, i64, i64, i64, vp, ci, ci, vp, i64, vp],
        "qcfg_quant_error_sweep": [vp, C.POINTER(vp), C.POINTER(i64), C.POINTER(i64), i32, ci, ci, ci, vp, vp, vp],
        "qcfg_quant_error_sweep_static": [vp, C.POINTER(vp), C.POINTER(i64), C.POINTER(i64), i32, ci, ci, ci, vp, vp, vp],
        "qcfg_gemm_i8": [vp, vp, i64, vp, i64, i64, i64, i64, f32, vp, ci, vp, vp, vp],
        "qcfg_gemm_i8_requant": [vp, vp, i64, vp, i64, i64, i64, i64, f32, vp, ci, f32, ci, vp, i64, vp],
        "qcfg_gemm_bf16": [vp, vp, i64, vp, i64, i64, i64, i64, ci, vp, vp],
        "qcfg_quantize_tokens": [vp, vp, ci, i64, i64, i64, ci, vp, i64, vp, vp],
        "qcfg_gemm_i8_token": [vp, vp, i64, vp, i64, i64, i64, i64, vp, vp, vp, ci, vp, ci, i64, vp],
        "qcfg_linear_i8": [vp, vp, ci, i64, ci, vp, i64, i64, i64, i64, vp, vp, ci, vp, ci, i64, vp, i64, vp],
        "qcfg_kv_extend": [vp, pool, batch, vp],
        "qcfg_kv_free": [vp, pool, vp, i32, vp],
        "qcfg_kv_fork": [vp, pool, vp, vp, i32, vp, vp, vp],
        "qcfg_kv_compact": [vp, pool, vp, vp],
        "qcfg_kv_copy_pages": [vp, pool, cache, vp, vp, i32, vp],
        "qcfg_kv_append": [vp, pool, cache, batch, vp, vp, ci, i64, i64, vp],
        "qcfg_kv_read": [vp, pool, cache, batch, vp, vp, vp, ci, vp],
        "qcfg_kv_attention": [vp, pool, cache, batch, vp, i64, i64, i32, vp, i64, i64, ci, i32, i32, f32, ci, i32, vp, i64, vp],
        "qcfg_model_create": [vp, C.POINTER(LayerStruct), i32, C.POINTER(vp)],
        "qcfg_model_set_attention": [vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, ci, i32],
        "qcfg_model_destroy": [vp],
        "qcfg_calibrate_model": [vp, vp, vp, i64, vp],
        "qcfg_model_act_absmax": [vp, C.POINTER(f32)],
        "qcfg_model_weight_absmax": [vp, i32, C.POINTER(f32)],
        "qcfg_eval_config": [vp, vp, C.POINTER(C.c_uint8), vp, i64, C.POINTER(vp), vp],
        "qcfg_debug_dump": [vp, vp, i32, vp, vp, vp, vp],
        "qcfg_debug_launch_forms": [vp, C.POINTER(i64)],
        "qcfg_search": [vp, vp, ci, C.POINTER(i32), C.POINTER(C.c_uint8), i32, C.c_double, vp, i64, C.POINTER(C.c_uint8),
                        C.POINTER(C.c_uint8), C.POINTER(C.c_double), i32, C.POINTER(i32), vp],
        "qcfg_noise_sensitivity": [vp, vp, vp, i64, C.POINTER(C.c_void_p), C.c_float, C.POINTER(C.c_double), vp],
        "qcfg_adjust_scales": [vp, vp, C.POINTER(C.c_uint8), vp, i64, i32, C.c_double, C.POINTER(C.c_double), vp],
        "qcfg_scale_gradients": [vp, vp, C.POINTER(C.c_uint8), vp, i64, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                 C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_double), vp],
        "qcfg_model_scales": [vp, i32, ci, C.POINTER(f32), C.POINTER(f32), C.POINTER(f32), C.POINTER(f32)],
        "qcfg_model_reset_scales": [vp],
        "qcfg_latency_table": [vp, vp, vp, i64, C.POINTER(C.c_uint8), i32, i32, C.POINTER(C.c_float), vp],
        "qcfg_config_cost": [vp, C.POINTER(C.c_uint8), C.POINTER(C.c_uint8), i32, C.POINTER(C.c_float), C.POINTER(C.c_double),
                             C.POINTER(C.c_double)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ci
    lib.qcfg_last_error.argtypes = [vp]
    lib.qcfg_last_error.restype = C.c_char_p
    lib.qcfg_launch_count.argtypes = [vp]
    lib.qcfg_launch_count.restype = i64
    lib.qcfg_linear_i8_work.argtypes = [i64, i64]
    lib.qcfg_linear_i8_work.restype = i64
    lib.qcfg_kv_attention_work.argtypes = [vp, cache, i64, i32]
    lib.qcfg_kv_attention_work.restype = i64
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _doubles(a) -> List[float]:
    """A ctypes array of doubles as a list (one conversion of the buffer, not one per element)."""
    return memoryview(a).cast("B").cast("d").tolist()


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


class Context:
    """Owns one qcfg_ctx.  Methods carry the C entry points' names without the prefix."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        h = C.c_void_p()
        rc = self.lib.qcfg_create(C.byref(h), device)
        if rc != OK:
            raise QcfgError(rc, "qcfg_create failed (an sm_100 CUDA device is required)")
        self.h = h
        self.device = device

    def close(self):
        if getattr(self, "h", None):
            self.lib.qcfg_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != OK:
            raise QcfgError(rc, self.last_error())

    def last_error(self) -> str:
        return self.lib.qcfg_last_error(self.h).decode()

    def launch_count(self) -> int:
        return int(self.lib.qcfg_launch_count(self.h))

    def launch_forms(self) -> dict:
        """GEMM launches of the context by the form they took (FORMS), since it was created."""
        counts = (C.c_int64 * len(FORMS))()
        self._check(self.lib.qcfg_debug_launch_forms(self.h, counts))
        return dict(zip(FORMS, counts))

    def sync_status(self, stream=None) -> int:
        return int(self.lib.qcfg_sync_status(self.h, _stream(stream)))

    def selftest_wait_timeout(self, limit_ns: int, stream=None):
        self._check(self.lib.qcfg_selftest_wait_timeout(self.h, int(limit_ns), _stream(stream)))

    def check_sync(self, stream=None):
        self._check(self.sync_status(stream))

    def set_fusion(self, enabled: bool):
        self._check(self.lib.qcfg_set_fusion(self.h, int(enabled)))

    def set_grouping(self, enabled: bool):
        self._check(self.lib.qcfg_set_grouping(self.h, int(enabled)))

    def set_prefix_reuse(self, enabled: bool):
        self._check(self.lib.qcfg_set_prefix_reuse(self.h, int(enabled)))

    def set_implicit_conv(self, enabled: bool):
        self._check(self.lib.qcfg_set_implicit_conv(self.h, int(enabled)))

    def set_gemm_chains(self, enabled: bool):
        self._check(self.lib.qcfg_set_gemm_chains(self.h, int(enabled)))

    def set_pair_tiles(self, enabled: bool):
        self._check(self.lib.qcfg_set_pair_tiles(self.h, int(enabled)))

    def profile_enable(self, mode):
        """0 off, 1 CUDA events around every launch, 2 in-kernel time stamps of the GEMM launches."""
        self._check(self.lib.qcfg_profile_enable(self.h, int(mode)))

    def profile_read(self, kernel_class: int, reset: bool = True):
        ms, n, ops = C.c_double(), C.c_int64(), C.c_double()
        self._check(self.lib.qcfg_profile_read(self.h, kernel_class, C.byref(ms), C.byref(n), C.byref(ops), int(reset)))
        return ms.value, n.value, ops.value

    # ---- tensor-level steps
    def calibrate(self, x: torch.Tensor, granularity: int, out: Optional[torch.Tensor] = None, stream=None):
        rows, cols = x.shape
        if out is None:
            out = torch.empty(1 if granularity == PER_TENSOR else rows, dtype=torch.float32, device=x.device)
        self._check(self.lib.qcfg_calibrate(self.h, _ptr(x), rows, cols, x.stride(0), granularity, _ptr(out), _stream(stream)))
        return out

    def scales_from_absmax(self, absmax: torch.Tensor, bits: int, stream=None):
        scale = torch.empty_like(absmax)
        inv = torch.empty_like(absmax)
        self._check(self.lib.qcfg_scales_from_absmax(self.h, _ptr(absmax), absmax.numel(), bits, _ptr(scale), _ptr(inv), _stream(stream)))
        return scale, inv

    def quantize(self, x: torch.Tensor, inv_scale: Optional[torch.Tensor], granularity: int, bits: int,
                 ldq: Optional[int] = None, stream=None) -> torch.Tensor:
        rows, cols = x.shape
        if ldq is None:
            ldq = (cols + 15) // 16 * 16
        q = torch.empty((rows, ldq), dtype=torch.bfloat16 if bits == 16 else torch.int8, device=x.device)
        self._check(self.lib.qcfg_quantize(self.h, _ptr(x), rows, cols, x.stride(0), _ptr(inv_scale), granularity, bits,
                                           _ptr(q), ldq, _stream(stream)))
        return q

    def quant_error_sweep(self, tensors: Sequence[torch.Tensor], granularity: int = PER_ROW, b_lo: int = 2, b_hi: int = 8,
                          sse: Optional[torch.Tensor] = None, absmax: Optional[torch.Tensor] = None, stream=None):
        n = len(tensors)
        nb = b_hi - b_lo + 1
        dev = tensors[0].device if n else torch.device("cuda", self.device)
        if sse is None:
            sse = torch.empty((n, nb), dtype=torch.float64, device=dev)
        if absmax is None:
            absmax = torch.empty(n, dtype=torch.float32, device=dev)
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in tensors])
        rows = (C.c_int64 * max(n, 1))(*[t.shape[0] for t in tensors])
        cols = (C.c_int64 * max(n, 1))(*[t.shape[1] for t in tensors])
        self._check(self.lib.qcfg_quant_error_sweep(self.h, ptrs, rows, cols, n, granularity, b_lo, b_hi, _ptr(sse),
                                                    _ptr(absmax), _stream(stream)))
        return sse, absmax

    def quant_error_sweep_static(self, tensors: Sequence[torch.Tensor], granularity: int = PER_ROW, b_lo: int = 2,
                                 b_hi: int = 8, sse: Optional[torch.Tensor] = None, absmax: Optional[torch.Tensor] = None,
                                 shapes: Optional[Sequence] = None, stream=None):
        """The sweep through the entry point that allocates no device memory (fixed scratch array
        inside the library, shared by all calls: do not overlap two of them on the GPU).  Pass
        `sse` and `absmax` to keep the binding from allocating either.  `shapes` overrides the
        (rows, cols) taken from the tensors."""
        n = len(tensors)
        nb = b_hi - b_lo + 1
        dev = tensors[0].device if n else torch.device("cuda", self.device)
        if sse is None:
            sse = torch.empty((n, nb), dtype=torch.float64, device=dev)
        if absmax is None:
            absmax = torch.empty(n, dtype=torch.float32, device=dev)
        shp = shapes if shapes is not None else [tuple(t.shape) for t in tensors]
        ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in tensors])
        rows = (C.c_int64 * max(n, 1))(*[s[0] for s in shp])
        cols = (C.c_int64 * max(n, 1))(*[s[1] for s in shp])
        self._check(self.lib.qcfg_quant_error_sweep_static(self.h, ptrs, rows, cols, n, granularity, b_lo, b_hi,
                                                           _ptr(sse), _ptr(absmax), _stream(stream)))
        return sse, absmax

    def gemm_i8(self, qx: torch.Tensor, qw: torch.Tensor, k: int, scale_x: float, scale_w: Optional[torch.Tensor],
                act: int = ACT_NONE, want_y: bool = True, want_acc: bool = False, stream=None):
        m, n = qx.shape[0], qw.shape[0]
        y = torch.empty((m, n), dtype=torch.float32, device=qx.device) if want_y else None
        acc = torch.empty((m, n), dtype=torch.int32, device=qx.device) if want_acc else None
        self._check(self.lib.qcfg_gemm_i8(self.h, _ptr(qx), qx.stride(0), _ptr(qw), qw.stride(0), m, n, k, scale_x,
                                          _ptr(scale_w), act, _ptr(y), _ptr(acc), _stream(stream)))
        return y, acc

    def gemm_i8_requant(self, qx: torch.Tensor, qw: torch.Tensor, k: int, scale_x: float, scale_w: torch.Tensor, act: int,
                        next_inv_scale: float, next_bits: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        m, n = qx.shape[0], qw.shape[0]
        if out is None:
            out = torch.zeros((m, (n + 15) // 16 * 16), dtype=torch.bfloat16 if next_bits == 16 else torch.int8, device=qx.device)
        self._check(self.lib.qcfg_gemm_i8_requant(self.h, _ptr(qx), qx.stride(0), _ptr(qw), qw.stride(0), m, n, k, scale_x,
                                                  _ptr(scale_w), act, next_inv_scale, next_bits, _ptr(out), out.stride(0),
                                                  _stream(stream)))
        return out

    def gemm_bf16(self, x: torch.Tensor, w: torch.Tensor, k: int, act: int = ACT_NONE, stream=None) -> torch.Tensor:
        m, n = x.shape[0], w.shape[0]
        y = torch.empty((m, n), dtype=torch.float32, device=x.device)
        self._check(self.lib.qcfg_gemm_bf16(self.h, _ptr(x), x.stride(0), _ptr(w), w.stride(0), m, n, k, act, _ptr(y), _stream(stream)))
        return y

    # ---- linear layers with a scale for each token
    def _on_device(self, *tensors):
        for t in tensors:
            if t is not None and t.get_device() != self.device:
                raise QcfgError(EINVAL, f"tensor on {t.device}, the context is on cuda:{self.device}")

    def quantize_tokens(self, x: torch.Tensor, bits: int = 8, ldq: Optional[int] = None, stream=None):
        """Codes of the rows of x (fp32, bf16 or fp16), each with its own scale.  Returns (codes [rows x ldq], scales)."""
        self._on_device(x)
        _rows_of(x)
        rows, cols = x.shape
        if ldq is None:
            ldq = (cols + 15) // 16 * 16
        q = _empty((rows, ldq), torch.int8, x.device, stream)
        scale = _empty(rows, torch.float32, x.device, stream)
        self._check(self.lib.qcfg_quantize_tokens(self.h, x.data_ptr(), _dtype(x.dtype), rows, cols, _ld(x), bits, q.data_ptr(), ldq,
                                                  scale.data_ptr(), self._here(stream)))
        return q, scale

    def gemm_i8_token(self, qx: torch.Tensor, qw: torch.Tensor, k: int, scale_x: torch.Tensor, scale_w: torch.Tensor,
                      bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, dtype: Optional[torch.dtype] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """act(float(qx qw^T) * (scale_x[m] * scale_w[n]) + bias[n]) as `dtype`: that of `out`, fp32 without one, unless given."""
        self._on_device(qx, qw, scale_x, scale_w, bias, out)
        for t in (qx, qw):
            _rows_of(t, torch.int8)
        m, n = qx.shape[0], qw.shape[0]
        if k > qx.shape[1] or k > qw.shape[1]:
            raise QcfgError(ESHAPE, "k is larger than the operands' rows")
        _vector(scale_x, m)
        _vector(scale_w, n)
        _vector(bias, n)
        out = _output(out, (m, n), dtype, torch.float32, qx.device, stream)
        self._check(self.lib.qcfg_gemm_i8_token(self.h, qx.data_ptr(), _ld(qx), qw.data_ptr(), _ld(qw), m, n, k, scale_x.data_ptr(),
                                                scale_w.data_ptr(), _at(bias), act, out.data_ptr(), _dtype(out.dtype), _ld(out),
                                                self._here(stream)))
        return out

    def linear_i8(self, x: torch.Tensor, qw: torch.Tensor, scale_w: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  act: int = ACT_NONE, bits: int = 8, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
        """A linear layer on x (fp32, bf16 or fp16, quantized row by row) with the weight codes qw [n x ld] that
        quantize(w, inv, PER_ROW, bits) gives and their scales.  `dtype` of the result: that of `out`, or of x, unless given."""
        self._on_device(x, qw, scale_w, bias, out)
        _rows_of(x)
        _rows_of(qw, torch.int8)
        (m, k), n = x.shape, qw.shape[0]
        if k > qw.shape[1]:
            raise QcfgError(ESHAPE, "x has more columns than the weight codes")
        _vector(scale_w, n)
        _vector(bias, n)
        out = _output(out, (m, n), dtype, x.dtype, x.device, stream)
        size = self.lib.qcfg_linear_i8_work(m, k)
        work = _empty(size, torch.uint8, x.device, stream) if size else None
        self._check(self.lib.qcfg_linear_i8(self.h, x.data_ptr(), _dtype(x.dtype), _ld(x), bits, qw.data_ptr(), _ld(qw), m, n, k,
                                            scale_w.data_ptr(), _at(bias), act, out.data_ptr(), _dtype(out.dtype), _ld(out), _at(work), size,
                                            self._here(stream)))
        return out

    def _here(self, stream) -> int:
        """The stream's handle; without one the current stream of the context's device."""
        return torch._C._cuda_getCurrentRawStream(self.device) if stream is None else stream.cuda_stream


def _rows_of(x: torch.Tensor, dtype: Optional[torch.dtype] = None):
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise QcfgError(ESHAPE, "a matrix with adjacent columns is needed")
    if dtype is not None and x.dtype != dtype:
        raise QcfgError(EINVAL, f"{dtype} is needed, got {x.dtype}")


def _ld(x: torch.Tensor) -> int:
    return x.stride(0) if x.shape[0] > 1 else max(x.shape[1], x.stride(0))


def _vector(x: Optional[torch.Tensor], n: int):
    if x is not None and (x.dtype != torch.float32 or x.numel() != n or not x.is_contiguous()):
        raise QcfgError(ESHAPE, f"{n} adjacent fp32 values are needed")


def _dtype(t: torch.dtype) -> int:
    if t not in DTYPES:
        raise QcfgError(EINVAL, f"fp32, bf16 or fp16 is needed, got {t}")
    return DTYPES[t]


def _empty(shape, dtype, device, stream):
    """Memory that belongs to the stream that will use it (None: the current one)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _output(out, shape, dtype, otherwise, device, stream):
    if out is None:
        dtype = dtype or otherwise
        _dtype(dtype)
        return _empty(shape, dtype, device, stream)
    if dtype is not None and out.dtype != dtype:
        raise QcfgError(EINVAL, f"out is {out.dtype}, {dtype} is asked for")
    if tuple(out.shape) != tuple(shape) or (out.shape[-1] > 1 and out.stride(-1) != 1):
        raise QcfgError(ESHAPE, f"out must be {tuple(shape)} with adjacent columns")
    return out


def _at(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _int32(x: Optional[torch.Tensor], n: Optional[int] = None):
    if x is not None and (x.dtype != torch.int32 or not x.is_contiguous() or (n is not None and x.numel() != n)):
        raise QcfgError(EINVAL, "adjacent int32 values are needed" + ("" if n is None else f", {n} of them"))


class KvPool:
    """Pages and the sequences that hold them (qcfg_kv_pool).  table [max_seqs, max_pages], lens [max_seqs] and refs [n_pages]
    are int32 tensors on the context's device, made here unless given.  refused [max_seqs]: 1 where the last extend with the sequence
    was refused; append leaves such sequences out."""

    def __init__(self, ctx: Context, n_pages: int, page_tokens: int, max_seqs: int, max_pages: int, table: Optional[torch.Tensor] = None,
                 lens: Optional[torch.Tensor] = None, refs: Optional[torch.Tensor] = None, refused: Optional[torch.Tensor] = None):
        dev = torch.device("cuda", ctx.device)
        self.ctx = ctx
        self.table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=dev) if table is None else table
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=dev) if lens is None else lens
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=dev) if refs is None else refs
        self.refused = torch.zeros(max_seqs, dtype=torch.int32, device=dev) if refused is None else refused
        ctx._on_device(self.table, self.lens, self.refs, self.refused)
        for t, n in ((self.table, max_seqs * max_pages), (self.lens, max_seqs), (self.refs, n_pages), (self.refused, max_seqs)):
            _int32(t, n)
        self.n_pages, self.page_tokens, self.max_seqs, self.max_pages = n_pages, page_tokens, max_seqs, max_pages
        self._c = PoolStruct(self.table.data_ptr(), self.lens.data_ptr(), self.refs.data_ptr(), n_pages, page_tokens, max_seqs, max_pages,
                             self.refused.data_ptr())
        self._ref = C.byref(self._c)

    def _batch(self, seqs: torch.Tensor, starts: Optional[torch.Tensor], rows: int):
        n = seqs.numel()
        _int32(seqs)
        self.ctx._on_device(seqs, starts)
        if starts is None:
            return C.byref(BatchStruct(seqs.data_ptr(), None, n, rows))
        _int32(starts, n + 1)
        return C.byref(BatchStruct(seqs.data_ptr(), starts.data_ptr(), n, rows))

    def extend(self, seqs: torch.Tensor, starts: Optional[torch.Tensor] = None, rows: Optional[int] = None, stream=None):
        """Every sequence of `seqs` gets room for its rows (starts[i+1] - starts[i]; one each without starts).  All or nothing: without
        room nothing changes, append leaves these sequences out, and EPAGE surfaces from sync_status."""
        ctx = self.ctx
        ctx._check(ctx.lib.qcfg_kv_extend(ctx.h, self._ref, self._batch(seqs, starts, 0x7fffffff - 4096 if rows is None else rows),
                                          ctx._here(stream)))

    def free(self, seqs: torch.Tensor, stream=None):
        ctx = self.ctx
        _int32(seqs)
        ctx._on_device(seqs)
        ctx._check(ctx.lib.qcfg_kv_free(ctx.h, self._ref, seqs.data_ptr(), seqs.numel(), ctx._here(stream)))

    def fork(self, parents: torch.Tensor, children: torch.Tensor, stream=None):
        """Returns (src, dst): the pages that copy_pages has to copy in every layer's cache."""
        ctx, n = self.ctx, parents.numel()
        _int32(parents)
        _int32(children, n)
        ctx._on_device(parents, children)
        src, dst = _empty((2, n), torch.int32, parents.device, stream).unbind()
        ctx._check(ctx.lib.qcfg_kv_fork(ctx.h, self._ref, parents.data_ptr(), children.data_ptr(), n, src.data_ptr(), dst.data_ptr(),
                                        ctx._here(stream)))
        return src, dst

    def compact(self, stream=None) -> torch.Tensor:
        """Returns the new number of every page in use, -1 for free ones: copy_pages(None, that) moves the contents."""
        ctx = self.ctx
        where = _empty(2 * self.n_pages, torch.int32, self.refs.device, stream)
        ctx._check(ctx.lib.qcfg_kv_compact(ctx.h, self._ref, where.data_ptr(), ctx._here(stream)))
        return where[:self.n_pages]


class KvCache:
    """One layer's keys and values in int8 (qcfg_kv_cache): codes [n_pages, kv_heads, page_tokens, head_dim] and maxima
    [n_pages, kv_heads], made here unless given."""

    def __init__(self, pool: KvPool, kv_heads: int, head_dim: int, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                 k_absmax: Optional[torch.Tensor] = None, v_absmax: Optional[torch.Tensor] = None):
        dev = torch.device("cuda", pool.ctx.device)
        self.pool, self.ctx, self.kv_heads, self.head_dim = pool, pool.ctx, kv_heads, head_dim
        shape = (pool.n_pages, kv_heads, pool.page_tokens, head_dim)
        self.k, self.v = (torch.zeros(shape, dtype=torch.int8, device=dev) if t is None else t for t in (k, v))
        self.k_absmax, self.v_absmax = (torch.zeros(shape[:2], dtype=torch.float32, device=dev) if t is None else t for t in (k_absmax, v_absmax))
        self.ctx._on_device(self.k, self.v, self.k_absmax, self.v_absmax)
        for t, want, dt in ((self.k, shape, torch.int8), (self.v, shape, torch.int8), (self.k_absmax, shape[:2], torch.float32),
                            (self.v_absmax, shape[:2], torch.float32)):
            if tuple(t.shape) != want or t.dtype != dt or not t.is_contiguous():
                raise QcfgError(ESHAPE, f"a dense {dt} tensor of {want} is needed")
        self._c = CacheStruct(self.k.data_ptr(), self.v.data_ptr(), self.k_absmax.data_ptr(), self.v_absmax.data_ptr(), kv_heads, head_dim)
        self._ref = C.byref(self._c)

    def _heads_of(self, x: torch.Tensor, heads: Optional[int]):
        if x.dim() != 3 or x.shape[2] != self.head_dim or x.stride(2) != 1 or (heads is not None and x.shape[1] != heads):
            raise QcfgError(ESHAPE, f"[rows, {heads or 'heads'}, {self.head_dim}] with adjacent elements is needed")

    def append(self, k: torch.Tensor, v: torch.Tensor, seqs: torch.Tensor, starts: Optional[torch.Tensor] = None, stream=None):
        """Writes the last tokens of every sequence of the batch (KvPool.extend has made room for them)."""
        ctx = self.ctx
        ctx._on_device(k, v)
        self._heads_of(k, self.kv_heads)
        self._heads_of(v, self.kv_heads)
        strides = k.stride()
        if k.shape != v.shape or k.dtype != v.dtype or any(n > 1 and a != b for n, a, b in zip(k.shape, strides, v.stride())):
            raise QcfgError(ESHAPE, "keys and values must agree in shape, type and strides")
        ctx._check(ctx.lib.qcfg_kv_append(ctx.h, self.pool._ref, self._ref, self.pool._batch(seqs, starts, k.shape[0]), k.data_ptr(),
                                          v.data_ptr(), _dtype(k.dtype), strides[0], strides[1], ctx._here(stream)))

    def read(self, seqs: torch.Tensor, first: torch.Tensor, starts: Optional[torch.Tensor], rows: int, dtype: torch.dtype = torch.float32,
             stream=None):
        """Values of the tokens first[i] .. of every sequence, as many as its rows: (k, v), each [rows, kv_heads, head_dim].
        Rows behind the last sequence's are left as they are (unset)."""
        ctx = self.ctx
        _int32(first, seqs.numel())
        ctx._on_device(first)
        kind = _dtype(dtype)
        k, v = _empty((2, rows, self.kv_heads, self.head_dim), dtype, self.k.device, stream).unbind()
        ctx._check(ctx.lib.qcfg_kv_read(ctx.h, self.pool._ref, self._ref, self.pool._batch(seqs, starts, rows), first.data_ptr(), k.data_ptr(),
                                        v.data_ptr(), kind, ctx._here(stream)))
        return k, v

    def copy_pages(self, src: Optional[torch.Tensor], dst: torch.Tensor, stream=None):
        """Page src[i] (i itself without src) to page dst[i]; entries of -1 are passed over."""
        ctx, n = self.ctx, dst.numel()
        _int32(dst)
        _int32(src, n)
        ctx._on_device(src, dst)
        ctx._check(ctx.lib.qcfg_kv_copy_pages(ctx.h, self.pool._ref, self._ref, _at(src), dst.data_ptr(), n, ctx._here(stream)))

    def attention(self, q: torch.Tensor, seqs: torch.Tensor, starts: Optional[torch.Tensor] = None, sm_scale: Optional[float] = None,
                  causal: bool = True, window: int = 0, max_new: int = 0, max_len: int = 0, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
        """softmax(sm_scale * q k^T) v of the last tokens of every sequence: q [rows, q_heads, head_dim], out like q.
        sm_scale: 1 / sqrt(head_dim) unless given; max_new, max_len: the longest entry and sequence, where known."""
        ctx, shape = self.ctx, q.shape
        ctx._on_device(q, out)
        self._heads_of(q, None)
        kind = _dtype(q.dtype)
        if out is None:
            out = _empty(shape, q.dtype, q.device, stream)
        elif out.dtype != q.dtype or out.shape != shape or out.stride(2) != 1:
            raise QcfgError(ESHAPE, "out must be like q, with adjacent elements")
        size = ctx.lib.qcfg_kv_attention_work(ctx.h, self._ref, shape[0], max_len)
        work = _empty(size, torch.uint8, q.device, stream) if size else None
        qs, os_ = q.stride(), out.stride()
        ctx._check(ctx.lib.qcfg_kv_attention(ctx.h, self.pool._ref, self._ref, self.pool._batch(seqs, starts, shape[0]), q.data_ptr(), qs[0], qs[1],
                                             shape[1], out.data_ptr(), os_[0], os_[1], kind, max_new, max_len,
                                             self.head_dim ** -0.5 if sm_scale is None else sm_scale, causal, window, _at(work), size,
                                             ctx._here(stream)))
        return out


class Model:
    """Owns one qcfg_model built from a list of layer descriptions and device weights."""

    def __init__(self, ctx: Context, layers, weights: Sequence[torch.Tensor]):
        self.ctx = ctx
        self.layers = list(layers)
        self.weights = list(weights)          # keeps the borrowed device memory alive
        arr = (LayerStruct * len(self.layers))()
        for i, (l, w) in enumerate(zip(self.layers, self.weights)):
            assert w.dtype == torch.float32 and w.is_contiguous() and tuple(w.shape) == (l.n_out, l.k_in)
            arr[i] = LayerStruct(w.data_ptr(), l.n_out, l.k_in, l.src, l.src_col0, l.act, l.kh, l.kw, l.stride, l.pad,
                                 l.in_h, l.in_w, l.in_c, l.pool_before, l.src_h, l.src_w, l.residual_from)
        h = C.c_void_p()
        ctx._check(ctx.lib.qcfg_model_create(ctx.h, arr, len(self.layers), C.byref(h)))
        self.h = h

    def close(self):
        if getattr(self, "h", None) and self.ctx.h:
            self.ctx.lib.qcfg_model_destroy(self.h)
        self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_attention(self, layer: int, k_layer: int, v_layer: int, q_heads: int, kv_heads: int, seq_len: int, page_tokens: int = 64,
                      sm_scale: Optional[float] = None, causal: bool = True, window: int = 0):
        """Layer `layer` reads the attention of its source's rows over k_layer's and v_layer's, keys and values held at 8 bits.
        sm_scale None: 1 / sqrt(head_dim)."""
        if sm_scale is None:
            sm_scale = (q_heads / max(self.layers[layer].k_in, 1)) ** 0.5 if 0 <= layer < len(self.layers) and q_heads > 0 else 1.0
        self.ctx._check(self.ctx.lib.qcfg_model_set_attention(self.ctx.h, self.h, layer, k_layer, v_layer, q_heads, kv_heads, seq_len,
                                                              page_tokens, sm_scale, int(causal), window))

    def calibrate_model(self, x: torch.Tensor, m: int, stream=None):
        self.ctx._check(self.ctx.lib.qcfg_calibrate_model(self.ctx.h, self.h, _ptr(x), m, _stream(stream)))

    def act_absmax(self) -> List[float]:
        out = (C.c_float * len(self.layers))()
        self.ctx._check(self.ctx.lib.qcfg_model_act_absmax(self.h, out))
        return list(out)

    def weight_absmax(self, layer: int):
        out = (C.c_float * self.layers[layer].n_out)()
        self.ctx._check(self.ctx.lib.qcfg_model_weight_absmax(self.h, layer, out))
        return list(out)

    def eval_config(self, bits, x: torch.Tensor, m: int, y: Optional[Sequence[Optional[torch.Tensor]]] = None, stream=None):
        n = len(self.layers)
        b = (C.c_uint8 * n)(*[int(v) for v in bits])
        yp = None
        if y is not None:
            yp = (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in y])
        self.ctx._check(self.ctx.lib.qcfg_eval_config(self.ctx.h, self.h, b, _ptr(x), m, yp, _stream(stream)))

    def search(self, algorithm: int, order, bs, target: float, x: torch.Tensor, m: int, capacity: int = 4096, stream=None):
        """Algorithm 1 (algorithm=0, bisection) or 2 (1, greedy).  Returns (bits, visited configurations, fidelities)."""
        n = len(self.layers)
        order_a = (C.c_int32 * n)(*[int(v) for v in order])
        bs_a = (C.c_uint8 * len(bs))(*[int(v) for v in bs])
        bits = (C.c_uint8 * n)()
        visited = (C.c_uint8 * (capacity * n))()
        acc = (C.c_double * capacity)()
        n_evals = C.c_int32()
        self.ctx._check(self.ctx.lib.qcfg_search(self.ctx.h, self.h, algorithm, order_a, bs_a, len(bs), float(target), _ptr(x), m,
                                                 bits, visited, acc, capacity, C.byref(n_evals), _stream(stream)))
        k = min(n_evals.value, capacity)
        vis = [list(visited[i * n:(i + 1) * n]) for i in range(k)]
        return list(bits), vis, list(acc[:k]), n_evals.value

    def noise_sensitivity(self, x: torch.Tensor, m: int, noises, lam: float, stream=None):
        """E_N per layer (Eqs. 3-5); noises[l] is a standard-normal tensor shaped like layer l's weight, or None."""
        n = len(self.layers)
        ptrs = (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in noises])
        out = (C.c_double * n)()
        self.ctx._check(self.ctx.lib.qcfg_noise_sensitivity(self.ctx.h, self.h, _ptr(x), m, ptrs, float(lam), out, _stream(stream)))
        return list(out)

    def adjust_scales(self, bits, x: torch.Tensor, m: int, steps: int, lr: float = 1e-5, stream=None):
        """Section 3.1's adjustment step: `steps` gradient steps on the scales.  Returns the losses (steps + 1)."""
        n = len(self.layers)
        b = (C.c_uint8 * n)(*[int(v) for v in bits])
        losses = (C.c_double * (steps + 1))()
        self.ctx._check(self.ctx.lib.qcfg_adjust_scales(self.ctx.h, self.h, b, _ptr(x), m, steps, float(lr), losses, _stream(stream)))
        return list(losses)

    def scale_gradients(self, bits, x: torch.Tensor, m: int, stream=None):
        """(loss, d_scale_x, d_inv_scale_x, d_scale_w, d_inv_scale_w); the last two are lists of per-channel lists."""
        n = len(self.layers)
        b = (C.c_uint8 * n)(*[int(v) for v in bits])
        dsx, dix, loss = (C.c_double * n)(), (C.c_double * n)(), C.c_double()
        bufs_s = [(C.c_double * l.n_out)() for l in self.layers]
        bufs_i = [(C.c_double * l.n_out)() for l in self.layers]
        ps = (C.c_void_p * n)(*[C.addressof(a) for a in bufs_s])
        pi = (C.c_void_p * n)(*[C.addressof(a) for a in bufs_i])
        self.ctx._check(self.ctx.lib.qcfg_scale_gradients(self.ctx.h, self.h, b, _ptr(x), m, dsx, dix, ps, pi, C.byref(loss), _stream(stream)))
        return loss.value, list(dsx), list(dix), [_doubles(a) for a in bufs_s], [_doubles(a) for a in bufs_i]

    def scales(self, layer: int, bits: int):
        """(scale_x, inv_scale_x, scale_w[n_out], inv_scale_w[n_out]) in use for `layer` at `bits`."""
        n_out = self.layers[layer].n_out
        sx, ix = C.c_float(), C.c_float()
        sw, iw = (C.c_float * n_out)(), (C.c_float * n_out)()
        self.ctx._check(self.ctx.lib.qcfg_model_scales(self.h, layer, bits, C.byref(sx), C.byref(ix), sw, iw))
        return sx.value, ix.value, list(sw), list(iw)

    def reset_scales(self):
        self.ctx._check(self.ctx.lib.qcfg_model_reset_scales(self.h))

    def latency_table(self, x: torch.Tensor, m: int, bs, reps: int = 5, stream=None):
        """Mean milliseconds of every layer at every width of bs: list of n_layers rows of len(bs) floats."""
        n = len(self.layers)
        bs_a = (C.c_uint8 * len(bs))(*[int(v) for v in bs])
        out = (C.c_float * (n * len(bs)))()
        self.ctx._check(self.ctx.lib.qcfg_latency_table(self.ctx.h, self.h, _ptr(x), m, bs_a, len(bs), reps, out, _stream(stream)))
        return [list(out[l * len(bs):(l + 1) * len(bs)]) for l in range(n)]

    def config_cost(self, bits, bs=None, table=None):
        """(latency in ms or None, size in bytes) of a configuration; latency needs bs and the table."""
        n = len(self.layers)
        b = (C.c_uint8 * n)(*[int(v) for v in bits])
        size = C.c_double()
        if table is None:
            self.ctx._check(self.ctx.lib.qcfg_config_cost(self.h, b, None, 0, None, None, C.byref(size)))
            return None, size.value
        bs_a = (C.c_uint8 * len(bs))(*[int(v) for v in bs])
        flat = (C.c_float * (n * len(bs)))(*[float(v) for row in table for v in row])
        lat = C.c_double()
        self.ctx._check(self.ctx.lib.qcfg_config_cost(self.h, b, bs_a, len(bs), flat, C.byref(lat), C.byref(size)))
        return lat.value, size.value

    def debug_dump(self, layer: int, qx: Optional[torch.Tensor], qw: Optional[torch.Tensor], acc: Optional[torch.Tensor], stream=None):
        self.ctx._check(self.ctx.lib.qcfg_debug_dump(self.ctx.h, self.h, layer, _ptr(qx), _ptr(qw), _ptr(acc), _stream(stream)))
