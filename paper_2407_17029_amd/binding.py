"""Thin ctypes binding over the C-ABI library (include/qblora.h), same entry-point names.

Argument marshalling only: PyTorch allocates device buffers and supplies the stream; every step
of the method runs inside libqblora.so.  There is no CPU fallback: if the library has not been
built (python -m paper_2407_17029_amd.build) loading raises, and every call checks the returned
status code and raises on error.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np
import torch

_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_DIR, "libqblora.so")

OK = 0
QUANT_ABSMAX_CODEBOOK, QUANT_MINMAX_INT4 = 0, 1
SCALES_FP32, SCALES_E4M3_GROUPED = 0, 1
MERGE_BETA_SHIFT, MERGE_REQUANT_MINMAX = 0, 1
OP_AVGPOOL_REPEAT, OP_TRUNCATE_PAD0, OP_SAMPLE_ZEROFILL = 0, 1, 2
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = 0, 1, 2, 3

EXPORTS = ["qblora_quantize_blockwise", "qblora_dequantize_bf16", "qblora_linear_fwd_workspace_bytes",
           "qblora_linear_bwd_workspace_bytes", "qblora_linear_fwd", "qblora_linear_bwd",
           "qblora_tile_product_workspace_bytes", "qblora_tile_product", "qablora_merge_quantize",
           "qablora_merge_quantize_batch",
           "qblora_strerror", "qblora_profile_events", "qblora_codes_tiled_bytes", "qblora_prepack_codes",
           "qblora_saved_bytes", "qblora_linear_fwd_save", "qblora_linear_bwd_saved",
           "qablora_linear_fwd_workspace_bytes", "qablora_linear_bwd_workspace_bytes", "qablora_linear_fwd",
           "qablora_linear_bwd", "qblora_merge_bf16",
           "qblora_linear_decode_workspace_bytes", "qblora_linear_decode_tokens_workspace_bytes", "qblora_linear_decode",
           "qblora_decode_pack_bytes", "qblora_decode_pack",
           "qblora_noalloc_scratch_bytes", "qblora_linear_fwd_noalloc", "qblora_dense_min_tokens",
           "qblora_page_tables", "qblora_rope_fwd", "qblora_rope_bwd", "qblora_rope_cache", "qblora_rope_frequencies",
           "qblora_paged_attention_workspace_bytes", "qblora_paged_attention", "qblora_rms_norm_fwd",
           "qblora_rms_norm_bwd_workspace_bytes", "qblora_rms_norm_bwd",
           "qblora_adapter_table_bytes", "qblora_adapter_table", "qblora_adapter_tiles", "qblora_adapter_groups",
           "qblora_adapters_saved_bytes", "qblora_adapters_workspace_bytes", "qblora_adapters_fwd", "qblora_adapters_bwd",
           "qblora_adamw_plan_bytes", "qblora_adamw_plan", "qblora_grad_norm_workspace_bytes", "qblora_grad_norm",
           "qblora_adamw_step"]

PROFILE_FWD_GEMM, PROFILE_BWD_GEMM, PROFILE_MERGE, PROFILE_QUANTIZE = 0, 1, 2, 3
PROFILE_ADAPTER_FWD, PROFILE_ADAPTER_BWD, PROFILE_ADAPTER_GRADS, PROFILE_GRAD_REDUCE = 4, 5, 6, 7
PROFILE_PREP, PROFILE_TILE_PRODUCT, PROFILE_DEQUANT = 8, 9, 10


class CQWeight(C.Structure):
    _fields_ = [("d_out", C.c_int32), ("d_in", C.c_int32), ("block", C.c_int32), ("scale_mode", C.c_int32),
                ("scale_group", C.c_int32), ("codebook", C.c_float * 16), ("codes", C.c_void_p),
                ("scales", C.c_void_p), ("beta", C.c_void_p), ("scale_codes", C.c_void_p),
                ("scale_step", C.c_void_p), ("scale_mid", C.c_void_p), ("codes_tiled", C.c_void_p),
                ("block_rows", C.c_int32)]


class CAdapter(C.Structure):
    _fields_ = [("lambda1", C.c_int32), ("lambda2", C.c_int32), ("R", C.c_int32), ("s", C.c_float),
                ("A", C.c_void_p), ("B", C.c_void_p), ("scale_op", C.c_int32)]


class CKVCache(C.Structure):
    _fields_ = [("pages", C.c_int32), ("page", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p)]


class CRope(C.Structure):
    _fields_ = [("rot", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float), ("freq", C.c_void_p)]


class CAdapters(C.Structure):
    _fields_ = [("count", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32), ("lambda1", C.c_int32),
                ("lambda2", C.c_int32), ("R", C.c_int32), ("table", C.c_void_p)]


class CAdamWTensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p),
                ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("rate", C.c_float), ("decay", C.c_float)]


class CAdamWList(C.Structure):
    _fields_ = [("count", C.c_int32), ("bits", C.c_int32), ("units", C.c_int64), ("plan", C.c_void_p)]


class CAdamW(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64),
                ("device_step", C.c_void_p), ("device_lr", C.c_void_p), ("seed", C.c_uint32)]


# The same layouts for struct.pack: one call instead of a descriptor access per field (a description of a weight took 9 us
# of the 10 that a small inference call spent in Python, now 2).
_QWEIGHT, _ADAPTER = struct.Struct("=5i64s4x7Qi4x"), struct.Struct("=3if2Qi4x")
_FLOAT32 = np.dtype(np.float32)
assert _QWEIGHT.size == C.sizeof(CQWeight) and _ADAPTER.size == C.sizeof(CAdapter)
_KV_CACHE, _ROPE = struct.Struct("=4i2Q"), struct.Struct("=2if4xQ")
assert _KV_CACHE.size == C.sizeof(CKVCache) and _ROPE.size == C.sizeof(CRope)
_ADAPTERS, _ADAMW = struct.Struct("=6iQ"), struct.Struct("=4dq2QI4x")
assert _ADAPTERS.size == C.sizeof(CAdapters) and _ADAMW.size == C.sizeof(CAdamW)


class QBLoRAError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


_lib = None


def lib():
    """Load libqblora.so (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_17029_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.qblora_strerror.restype = C.c_char_p
        L.qblora_strerror.argtypes = [C.c_int]
        for name in ("qblora_linear_fwd_workspace_bytes", "qblora_linear_bwd_workspace_bytes",
                     "qblora_tile_product_workspace_bytes"):
            getattr(L, name).restype = C.c_size_t
        L.qblora_linear_fwd_workspace_bytes.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.qblora_linear_bwd_workspace_bytes.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.qblora_tile_product_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        L.qblora_quantize_blockwise.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                                C.c_int32, C.c_void_p, C.c_void_p]
        L.qblora_dequantize_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.qblora_linear_fwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                        C.c_size_t, C.c_void_p]
        L.qblora_linear_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.qblora_tile_product.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t,
                                          C.c_void_p]
        L.qablora_merge_quantize.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_int32,
                                             C.c_void_p, C.c_void_p]
        L.qablora_merge_quantize_batch.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float,
                                                   C.c_int32, C.c_void_p, C.c_void_p]
        L.qblora_profile_events.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]
        L.qblora_codes_tiled_bytes.restype = C.c_size_t
        L.qblora_codes_tiled_bytes.argtypes = [C.c_int32, C.c_int32]
        L.qblora_prepack_codes.argtypes = [C.c_void_p, C.c_void_p]
        for name in ("qablora_linear_fwd_workspace_bytes", "qablora_linear_bwd_workspace_bytes"):
            getattr(L, name).restype = C.c_size_t
            getattr(L, name).argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int64]
        L.qablora_linear_fwd.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.qablora_linear_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p,
                                         C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.qblora_merge_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p]
        L.qblora_linear_decode_workspace_bytes.restype = C.c_size_t
        L.qblora_linear_decode_workspace_bytes.argtypes = [C.c_void_p]
        L.qblora_linear_decode_tokens_workspace_bytes.restype = C.c_size_t
        L.qblora_linear_decode_tokens_workspace_bytes.argtypes = [C.c_void_p, C.c_int32]
        L.qblora_linear_decode.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t,
                                           C.c_void_p]
        L.qblora_decode_pack_bytes.restype = C.c_size_t
        L.qblora_decode_pack_bytes.argtypes = [C.c_void_p]
        L.qblora_decode_pack.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.qblora_saved_bytes.restype = C.c_size_t
        L.qblora_saved_bytes.argtypes = [C.c_void_p, C.c_int64]
        L.qblora_linear_fwd_save.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_size_t, C.c_void_p]
        L.qblora_linear_bwd_saved.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.qblora_dense_min_tokens.restype = C.c_int64
        L.qblora_dense_min_tokens.argtypes = []
        p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.qblora_page_tables.argtypes = [p, p, i32, i32, p, i32, p, i32, i64, p, p, p, p, p]
        for name in ("qblora_rope_fwd", "qblora_rope_bwd"):
            getattr(L, name).argtypes = [p, p, i64, i32, p, i64, i32, i32, p, i64, p, i64, p, i64, p]
        L.qblora_rope_cache.argtypes = [p, p, i64, i32, p, i64, p, i64, p, p, i64, p, i64, p, p]
        L.qblora_rope_frequencies.argtypes = [i32, C.c_double, i32, C.c_double, C.c_double, C.c_double, C.c_double, p, p]
        L.qblora_paged_attention_workspace_bytes.restype = C.c_size_t
        L.qblora_paged_attention_workspace_bytes.argtypes = [p, i32, i32]
        L.qblora_paged_attention.argtypes = [p, i64, i32, p, p, i32, p, p, i32, i64, C.c_float, i32, i32, p, i64, p, p,
                                             C.c_size_t, p]
        L.qblora_rms_norm_fwd.argtypes = [p, p, p, i64, i32, C.c_float, p, p, p, p]
        L.qblora_rms_norm_bwd_workspace_bytes.restype = C.c_size_t
        L.qblora_rms_norm_bwd_workspace_bytes.argtypes = [i64, i32]
        L.qblora_rms_norm_bwd.argtypes = [p, p, p, p, p, i64, i32, p, p, p, C.c_size_t, p]
        for name in ("qblora_adapter_table_bytes", "qblora_adapters_saved_bytes", "qblora_adapters_workspace_bytes",
                     "qblora_adamw_plan_bytes", "qblora_grad_norm_workspace_bytes"):
            getattr(L, name).restype = C.c_size_t
        L.qblora_adapter_table_bytes.argtypes = [i32]
        L.qblora_adapter_table.argtypes = [p, i32, i32, p, p, p, p]
        L.qblora_adapter_tiles.argtypes = [i32, i64]
        L.qblora_adapter_groups.argtypes = [p, p, i32, i32, i64, p, p, p, p]
        L.qblora_adapters_saved_bytes.argtypes = L.qblora_adapters_workspace_bytes.argtypes = [p, i64]
        L.qblora_adapters_fwd.argtypes = [p, p, p, p, p, i64, i64, p, i64, p, p, C.c_size_t, p]
        L.qblora_adapters_bwd.argtypes = [p, p, p, p, p, i64, p, i64, i64, p, p, i64, i32, p, C.c_size_t, p]
        L.qblora_adamw_plan_bytes.argtypes = [p, i32]
        L.qblora_adamw_plan.argtypes = [p, i32, i32, p, C.c_size_t, p, p]
        L.qblora_grad_norm_workspace_bytes.argtypes = [p]
        L.qblora_grad_norm.argtypes = [p, C.c_double, p, p, C.c_size_t, p]
        L.qblora_adamw_step.argtypes = [p, p, p, p]
        L.qblora_noalloc_scratch_bytes.restype = C.c_size_t
        L.qblora_noalloc_scratch_bytes.argtypes = []
        L.qblora_linear_fwd_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        _lib = L
    return _lib


_hip = None


def _hip_runtime():
    """The HIP runtime the process already uses (torch has loaded it)."""
    global _hip
    if _hip is None:
        _hip = C.CDLL("libamdhip64.so")
        _hip.hipEventCreateWithFlags.argtypes = [C.POINTER(C.c_void_p), C.c_uint]
        _hip.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        _hip.hipEventRecord.argtypes = [C.c_void_p, C.c_void_p]
        _hip.hipEventDestroy.argtypes = [C.c_void_p]
    return _hip


class TimingEvent:
    """A HIP event that only measures time: created with hipEventDisableSystemFence, i.e. without the
    system-scope cache write-back and invalidation an ordinary event record performs (which costs stream time
    and slows the kernel behind it).  Read it only after the stream has been synchronized by other means."""
    DISABLE_SYSTEM_FENCE = 0x20000000

    def __init__(self):
        h = C.c_void_p()
        if _hip_runtime().hipEventCreateWithFlags(C.byref(h), self.DISABLE_SYSTEM_FENCE) != 0:
            raise RuntimeError("hipEventCreateWithFlags failed")
        self.cuda_event = h.value

    def record(self, stream=None):
        if _hip_runtime().hipEventRecord(self.cuda_event, _stream() if stream is None else stream) != 0:
            raise RuntimeError("hipEventRecord failed")

    def elapsed_time(self, stop: "TimingEvent") -> float:
        ms = C.c_float()
        if _hip_runtime().hipEventElapsedTime(C.byref(ms), self.cuda_event, stop.cuda_event) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return float(ms.value)

    def __del__(self):
        try:
            _hip_runtime().hipEventDestroy(self.cuda_event)
        except Exception:
            pass


def qblora_profile_events(which: int, start=None, stop=None) -> None:
    """Register (or with None, unregister) a pair of timing events recorded around one kernel.

    `start` / `stop`: TimingEvent, or torch.cuda.Event created with enable_timing=True and recorded once
    already so that its native handle exists.
    """
    a = None if start is None else C.c_void_p(start.cuda_event)
    b = None if stop is None else C.c_void_p(stop.cuda_event)
    _check(lib().qblora_profile_events(which, a, b), "qblora_profile_events")


def strerror(code: int) -> str:
    return lib().qblora_strerror(code).decode()


def _check(code: int, where: str) -> None:
    if code != OK:
        raise QBLoRAError(code, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # without a torch.cuda.Stream object around it


def _stream():
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


class QWeight:
    """The triplet (codes, alpha, beta) of Eq. 1 on the device, plus the host-side C struct."""

    def __init__(self, d_out, d_in, block, codebook, codes, scales, beta=None, scale_mode=SCALES_FP32,
                 scale_codes=None, scale_step=None, scale_mid=None, scale_group=256, codes_tiled=None, block_rows=1):
        self.d_out, self.d_in, self.block = d_out, d_in, block
        self.block_rows = int(block_rows)       # 1: blocks of 64 inputs in a row; 8: blocks of 8 rows x 8 inputs
        self.codebook = np.asarray(codebook, np.float32)
        self.codes, self.scales, self.beta = codes, scales, beta
        self.scale_mode, self.scale_group = scale_mode, scale_group
        self.scale_codes, self.scale_step, self.scale_mid = scale_codes, scale_step, scale_mid
        self.codes_tiled = codes_tiled          # optional tile-ordered copy of the codes (forward fast path)

    def c_bytes(self) -> bytes:
        """The C struct as an immutable argument for calls that only read it; describes the object as it is now."""
        try:
            cb = self.codebook
            raw = cb.tobytes() if cb.dtype is _FLOAT32 and cb.shape == (16,) else bytes(self._c_struct())[20:84]
            return _QWEIGHT.pack(self.d_out, self.d_in, self.block, self.scale_mode, self.scale_group, raw, *[
                0 if t is None else t.data_ptr()
                for t in (self.codes, self.scales, self.beta, self.scale_codes, self.scale_step, self.scale_mid,
                          self.codes_tiled)], self.block_rows)
        except (struct.error, AttributeError):            # numbers and codebooks that only the fields themselves convert
            return bytes(self._c_struct())

    def c_struct(self) -> CQWeight:
        return CQWeight.from_buffer_copy(self.c_bytes())

    def _c_struct(self) -> CQWeight:
        s = CQWeight()
        s.d_out, s.d_in, s.block = self.d_out, self.d_in, self.block
        s.scale_mode, s.scale_group = self.scale_mode, self.scale_group
        s.block_rows = self.block_rows
        for j in range(16):
            s.codebook[j] = float(self.codebook[j])
        for name in ("codes", "scales", "beta", "scale_codes", "scale_step", "scale_mid", "codes_tiled"):
            t = getattr(self, name)
            setattr(s, name, None if t is None else t.data_ptr())
        return s

    def absorb(self, s: CQWeight) -> None:
        """Take back the scalar fields the library filled in."""
        self.d_out, self.d_in, self.block = s.d_out, s.d_in, s.block
        self.scale_mode, self.scale_group = s.scale_mode, s.scale_group
        self.codebook = np.array(s.codebook, np.float32)
        if not s.beta:
            self.beta = None


class Adapter:
    """Balanced adapter of Sec. 3.2: A bf16 [d_in/lambda1, R], B bf16 [R, d_out/lambda2], scaling s."""

    def __init__(self, A, B, lambda1, lambda2, s, scale_op=0):
        self.A, self.B, self.lambda1, self.lambda2, self.s = A, B, int(lambda1), int(lambda2), float(s)
        self.R = 0 if A is None else int(A.shape[1])
        self.scale_op = int(scale_op)        # OP_*: the scale operators of the ablation (Sec. 4.3)

    def c_bytes(self) -> bytes:
        """The C struct as an immutable argument, as of now."""
        try:
            return _ADAPTER.pack(self.lambda1, self.lambda2, self.R, self.s, 0 if self.A is None else self.A.data_ptr(),
                                 0 if self.B is None else self.B.data_ptr(), self.scale_op)
        except (struct.error, OverflowError):             # numbers that only the fields themselves convert
            return bytes(self.c_struct())

    def c_struct(self) -> CAdapter:
        a = CAdapter()
        a.lambda1, a.lambda2, a.R, a.s = self.lambda1, self.lambda2, self.R, self.s
        a.scale_op = self.scale_op
        a.A = None if self.A is None else self.A.data_ptr()
        a.B = None if self.B is None else self.B.data_ptr()
        return a


def _adapter(ad):
    return None if ad is None else ad.c_bytes()


def qblora_codes_tiled_bytes(d_out: int, d_in: int) -> int:
    return int(lib().qblora_codes_tiled_bytes(d_out, d_in))


def qblora_prepack_codes(qw: QWeight) -> QWeight:
    """Fill (allocating if needed) the tile-ordered copy of the codes from the reference layout."""
    if qw.codes_tiled is None:
        qw.codes_tiled = torch.empty(qblora_codes_tiled_bytes(qw.d_out, qw.d_in), dtype=torch.uint8,
                                     device=qw.codes.device)
    _check(lib().qblora_prepack_codes(qw.c_bytes(), _stream()), "qblora_prepack_codes")
    return qw


def qblora_quantize_blockwise(W: torch.Tensor, block: int = 64, quantizer: int = QUANT_ABSMAX_CODEBOOK,
                              codebook=None, scale_mode: int = SCALES_FP32, out: QWeight = None,
                              tiled: bool = True, block_rows: int = 1) -> QWeight:
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.dim() == 2
    d_out, d_in = W.shape
    dev = W.device
    if out is not None:                      # reuse the caller's buffers
        cb = np.zeros(16, np.float32) if codebook is None else np.ascontiguousarray(codebook, np.float32)
        s = out.c_struct()
        cb_ptr = None if codebook is None else cb.ctypes.data_as(C.c_void_p)
        rc = lib().qblora_quantize_blockwise(_ptr(W), d_out, d_in, block, quantizer, cb_ptr, scale_mode,
                                             C.byref(s), _stream())
        _check(rc, "qblora_quantize_blockwise")
        out.absorb(s)
        return out
    nblk = d_out * (d_in // max(block, 1))
    codes = torch.empty((d_out, d_in // 2), dtype=torch.uint8, device=dev)
    if block_rows == 8:                      # blocks of 8 rows x (block / 8) inputs: 8 x 8, or 8 x 4 with block = 32
        scales = torch.empty((d_out // 8, d_in // (block // 8)), dtype=torch.float32, device=dev)
    else:
        scales = torch.empty((d_out, d_in // max(block, 1)), dtype=torch.float32, device=dev)
    beta = torch.empty_like(scales) if quantizer == QUANT_MINMAX_INT4 else None
    sc = st = mid = None
    if scale_mode == SCALES_E4M3_GROUPED:
        ng = (nblk + 255) // 256
        sc = torch.empty(nblk, dtype=torch.uint8, device=dev)
        st = torch.empty(ng, dtype=torch.float32, device=dev)
        mid = torch.empty(ng, dtype=torch.float32, device=dev)
    cb = np.zeros(16, np.float32) if codebook is None else np.ascontiguousarray(codebook, np.float32)
    ct = None
    if tiled and block == 64 and d_in % 64 == 0:
        ct = torch.empty(qblora_codes_tiled_bytes(d_out, d_in), dtype=torch.uint8, device=dev)
    qw = QWeight(d_out, d_in, block, cb, codes, scales, beta, scale_mode, sc, st, mid, codes_tiled=ct,
                 block_rows=block_rows)
    s = qw.c_struct()
    cb_ptr = None if codebook is None else cb.ctypes.data_as(C.c_void_p)
    rc = lib().qblora_quantize_blockwise(_ptr(W), d_out, d_in, block, quantizer, cb_ptr, scale_mode, C.byref(s),
                                         _stream())
    _check(rc, "qblora_quantize_blockwise")
    qw.absorb(s)
    return qw


def qblora_dequantize_bf16(qw: QWeight) -> torch.Tensor:
    Wt = torch.empty((qw.d_out, qw.d_in), dtype=torch.bfloat16, device=qw.codes.device)
    _check(lib().qblora_dequantize_bf16(qw.c_bytes(), _ptr(Wt), _stream()), "qblora_dequantize_bf16")
    return Wt


def qblora_linear_fwd_workspace_bytes(qw: QWeight, ad, T: int) -> int:
    return int(lib().qblora_linear_fwd_workspace_bytes(qw.c_bytes(), _adapter(ad), T))


def qblora_linear_bwd_workspace_bytes(qw: QWeight, ad, T: int) -> int:
    return int(lib().qblora_linear_bwd_workspace_bytes(qw.c_bytes(), _adapter(ad), T))


def _workspace(nbytes, device, workspace):
    """The caller's workspace, or one of nbytes() bytes (a query that is only made when it is needed)."""
    if workspace is not None:
        return workspace
    return torch.empty(max(int(nbytes()), 256), dtype=torch.uint8, device=device)


def qblora_saved_bytes(ad, T: int) -> int:
    return int(lib().qblora_saved_bytes(_adapter(ad), T))


def qblora_linear_fwd(qw: QWeight, ad, X: torch.Tensor, Y: torch.Tensor = None, workspace: torch.Tensor = None,
                      saved: torch.Tensor = None):
    """`saved` (uint8 tensor of qblora_saved_bytes()) selects qblora_linear_fwd_save."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and X.shape[1] == qw.d_in
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, qw.d_out), dtype=torch.bfloat16, device=X.device)
    ws = _workspace(lambda: qblora_linear_fwd_workspace_bytes(qw, ad, T), X.device, workspace)
    s, a = qw.c_bytes(), _adapter(ad)
    if saved is None:
        rc = lib().qblora_linear_fwd(s, a, _ptr(X), T, _ptr(Y), _ptr(ws), ws.numel(), _stream())
        _check(rc, "qblora_linear_fwd")
    else:
        assert saved.is_cuda and saved.numel() * saved.element_size() >= lib().qblora_saved_bytes(a, T)
        rc = lib().qblora_linear_fwd_save(s, a, _ptr(X), T, _ptr(Y), _ptr(saved), _ptr(ws), ws.numel(),
                                          _stream())
        _check(rc, "qblora_linear_fwd_save")
    return Y


def qblora_dense_min_tokens() -> int:
    return int(lib().qblora_dense_min_tokens())


def qblora_noalloc_scratch_bytes() -> int:
    return int(lib().qblora_noalloc_scratch_bytes())


def qblora_linear_fwd_noalloc(qw: QWeight, ad, X: torch.Tensor, Y: torch.Tensor):
    """qblora_linear_fwd on the library's own scratch array: the caller passes inputs and the output only."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and X.shape[1] == qw.d_in
    assert Y.is_cuda and Y.dtype == torch.bfloat16 and Y.is_contiguous() and tuple(Y.shape) == (X.shape[0], qw.d_out)
    _check(lib().qblora_linear_fwd_noalloc(qw.c_bytes(), _adapter(ad), _ptr(X), X.shape[0], _ptr(Y), _stream()),
           "qblora_linear_fwd_noalloc")
    return Y


def qblora_linear_bwd(qw: QWeight, ad, X: torch.Tensor, dY: torch.Tensor, need_dx: bool = True,
                      need_grads: bool = True, dX=None, dA=None, dB=None, workspace: torch.Tensor = None,
                      saved: torch.Tensor = None):
    """`saved` (the buffer a forward call filled) selects qblora_linear_bwd_saved."""
    assert dY.is_cuda and dY.dtype == torch.bfloat16 and dY.is_contiguous() and dY.shape[1] == qw.d_out
    T = dY.shape[0]
    dev = dY.device
    if need_dx and dX is None:
        dX = torch.empty((T, qw.d_in), dtype=torch.bfloat16, device=dev)
    if need_grads and ad is not None and ad.R > 0:
        if dA is None:
            dA = torch.empty((qw.d_in // ad.lambda1, ad.R), dtype=torch.float32, device=dev)
        if dB is None:
            dB = torch.empty((ad.R, qw.d_out // ad.lambda2), dtype=torch.float32, device=dev)
    ws = _workspace(lambda: qblora_linear_bwd_workspace_bytes(qw, ad, T), dev, workspace)
    s, a = qw.c_bytes(), _adapter(ad)
    if saved is None:
        rc = lib().qblora_linear_bwd(s, a, _ptr(X), _ptr(dY), T, _ptr(dX), _ptr(dA), _ptr(dB), _ptr(ws),
                                     ws.numel(), _stream())
        _check(rc, "qblora_linear_bwd")
    else:
        rc = lib().qblora_linear_bwd_saved(s, a, _ptr(X), _ptr(dY), T, _ptr(saved), _ptr(dX), _ptr(dA),
                                           _ptr(dB), _ptr(ws), ws.numel(), _stream())
        _check(rc, "qblora_linear_bwd_saved")
    return dX, dA, dB


def qablora_linear_fwd(qw: QWeight, H: torch.Tensor, lambda1: int, lambda2: int, s: float, X: torch.Tensor,
                       Y: torch.Tensor = None, workspace: torch.Tensor = None):
    """Single-matrix adapter forward; H is bf16 [d_in/lambda1, d_out/lambda2]."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and X.shape[1] == qw.d_in
    assert H.is_cuda and H.dtype == torch.bfloat16 and H.is_contiguous()
    assert tuple(H.shape) == (qw.d_in // lambda1, qw.d_out // lambda2)
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, qw.d_out), dtype=torch.bfloat16, device=X.device)
    q = qw.c_bytes()
    ws = _workspace(lambda: lib().qablora_linear_fwd_workspace_bytes(q, lambda1, lambda2, T), X.device, workspace)
    rc = lib().qablora_linear_fwd(q, _ptr(H), lambda1, lambda2, s, _ptr(X), T, _ptr(Y), _ptr(ws), ws.numel(),
                                  _stream())
    _check(rc, "qablora_linear_fwd")
    return Y


def qablora_linear_bwd(qw: QWeight, H: torch.Tensor, lambda1: int, lambda2: int, s: float, X: torch.Tensor,
                       dY: torch.Tensor, need_dx: bool = True, need_dh: bool = True, dX=None, dH=None,
                       workspace: torch.Tensor = None):
    assert dY.is_cuda and dY.dtype == torch.bfloat16 and dY.is_contiguous() and dY.shape[1] == qw.d_out
    assert H.is_cuda and H.dtype == torch.bfloat16 and H.is_contiguous()
    T = dY.shape[0]
    dev = dY.device
    if need_dx and dX is None:
        dX = torch.empty((T, qw.d_in), dtype=torch.bfloat16, device=dev)
    if need_dh and dH is None:
        dH = torch.empty((qw.d_in // lambda1, qw.d_out // lambda2), dtype=torch.float32, device=dev)
    q = qw.c_bytes()
    ws = _workspace(lambda: lib().qablora_linear_bwd_workspace_bytes(q, lambda1, lambda2, T), dev, workspace)
    rc = lib().qablora_linear_bwd(q, _ptr(H), lambda1, lambda2, s, _ptr(X), _ptr(dY), T,
                                  _ptr(dX if need_dx else None), _ptr(dH if need_dh else None), _ptr(ws), ws.numel(),
                                  _stream())
    _check(rc, "qablora_linear_bwd")
    return (dX if need_dx else None), (dH if need_dh else None)


def qblora_tile_product(ad: Adapter, d_in: int, d_out: int, H: torch.Tensor = None, workspace=None):
    dev = ad.A.device
    if H is None:
        H = torch.empty((d_in // ad.lambda1, d_out // ad.lambda2), dtype=torch.float32, device=dev)
    a = ad.c_bytes()
    ws = _workspace(lambda: lib().qblora_tile_product_workspace_bytes(a, d_in, d_out), dev, workspace)
    rc = lib().qblora_tile_product(a, d_in, d_out, _ptr(H), _ptr(ws), ws.numel(), _stream())
    _check(rc, "qblora_tile_product")
    return H


def qablora_merge_quantize(base: QWeight, H: torch.Tensor, lambda1: int, lambda2: int, s: float, mode: int,
                           out: QWeight = None) -> QWeight:
    assert H.is_cuda and H.dtype == torch.float32 and H.is_contiguous()
    dev = H.device
    if out is None:
        out = QWeight(base.d_out, base.d_in, base.block, base.codebook,
                      torch.empty_like(base.codes),
                      torch.empty(tuple(base.scales.shape), dtype=torch.float32, device=dev),
                      torch.empty(tuple(base.scales.shape), dtype=torch.float32, device=dev),
                      block_rows=base.block_rows)
    o = out.c_struct()
    rc = lib().qablora_merge_quantize(base.c_bytes(), _ptr(H), lambda1, lambda2, s, mode, C.byref(o), _stream())
    _check(rc, "qablora_merge_quantize")
    beta_keep = out.beta
    out.absorb(o)
    out.beta = beta_keep
    out.scale_codes = out.scale_step = out.scale_mid = None
    out.codes_tiled = None
    return out


def qablora_merge_quantize_batch(bases, Hs, lambda1: int, lambda2: int, s: float, mode: int, outs=None):
    """qablora_merge_quantize for a list of weights (one launch per 8 where the kernels allow it)."""
    n = len(bases)
    assert len(Hs) == n and all(H.is_cuda and H.dtype == torch.float32 and H.is_contiguous() for H in Hs)
    if outs is None:
        outs = [QWeight(b.d_out, b.d_in, b.block, b.codebook, torch.empty_like(b.codes),
                        torch.empty(tuple(b.scales.shape), dtype=torch.float32, device=b.codes.device),
                        torch.empty(tuple(b.scales.shape), dtype=torch.float32, device=b.codes.device),
                        block_rows=b.block_rows) for b in bases]
    bs = (CQWeight * n).from_buffer_copy(b"".join([b.c_bytes() for b in bases]))
    os_ = (CQWeight * n).from_buffer_copy(b"".join([o.c_bytes() for o in outs]))
    barr, oarr = ((C.c_void_p * n)(*[C.addressof(a) + i * _QWEIGHT.size for i in range(n)]) for a in (bs, os_))
    harr = (C.c_void_p * n)(*[_ptr(H) for H in Hs])
    rc = lib().qablora_merge_quantize_batch(n, barr, harr, lambda1, lambda2, C.c_float(s), mode, oarr, _stream())
    _check(rc, "qablora_merge_quantize_batch")
    for o, oc in zip(outs, os_):
        beta_keep = o.beta
        o.absorb(oc)
        o.beta = beta_keep
        o.scale_codes = o.scale_step = o.scale_mid = None
        o.codes_tiled = None
    return outs


def qblora_merge_bf16(base: QWeight, H: torch.Tensor, lambda1: int, lambda2: int, s: float,
                      W16: torch.Tensor = None) -> torch.Tensor:
    """16-bit merge: bf16 [d_out, d_in] = w~ + s*dW."""
    assert H.is_cuda and H.dtype == torch.float32 and H.is_contiguous()
    if W16 is None:
        W16 = torch.empty((base.d_out, base.d_in), dtype=torch.bfloat16, device=H.device)
    rc = lib().qblora_merge_bf16(base.c_bytes(), _ptr(H), lambda1, lambda2, s, _ptr(W16), _stream())
    _check(rc, "qblora_merge_bf16")
    return W16


def qblora_decode_pack(qw: QWeight) -> torch.Tensor:
    """One-off tile-ordered copy of codes / scales / offsets for qblora_linear_decode."""
    q = qw.c_bytes()
    pack = torch.empty(int(lib().qblora_decode_pack_bytes(q)), dtype=torch.uint8, device=qw.codes.device)
    _check(lib().qblora_decode_pack(q, _ptr(pack), _stream()), "qblora_decode_pack")
    return pack


def qblora_linear_decode(qw: QWeight, X: torch.Tensor, Y: torch.Tensor = None, workspace: torch.Tensor = None,
                         pack: torch.Tensor = None):
    """Small- and mid-batch (T <= 256) forward of a quantized layer without adapter."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and X.shape[1] == qw.d_in
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, qw.d_out), dtype=torch.bfloat16, device=X.device)
    q = qw.c_bytes()
    ws = _workspace(lambda: lib().qblora_linear_decode_tokens_workspace_bytes(q, T), X.device, workspace)
    rc = lib().qblora_linear_decode(q, _ptr(pack), _ptr(X), T, _ptr(Y), _ptr(ws), ws.numel(), _stream())
    _check(rc, "qblora_linear_decode")
    return Y


# ---- between the projections of a decoder layer ---------------------------------------------------------
#
# These calls take a few microseconds on the GPU while a batch decodes, less than careless marshalling costs: each tensor is
# looked at once, and what is made here is not looked at again.

_BF16, _F32, _I32, _I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


def _address(t, dtype, shape) -> int:
    """Of a contiguous device array of this type and shape."""
    assert t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous()
    return t.data_ptr()


def _current_stream():
    return _stream() if _raw_stream is None else _raw_stream(torch._C._cuda_getDevice())


def _heads(t, T, heads, dim) -> int:
    """Elements from one token of a bf16 [T, heads, dim] to the next: any number, heads one behind the other."""
    assert t.dtype is _BF16 and t.is_cuda and t.shape == (T, heads, dim)
    if t.is_contiguous():
        return heads * dim
    token, head, feature = t.stride()
    assert (feature == 1 or dim == 1) and (head == dim or heads == 1)
    return token if T > 1 else max(token, heads * dim)


def _cache(k_cache, v_cache) -> bytes:
    """The description of a paged cache: keys [pages, heads, head_dim / 8, page, 8], values [pages, heads, page / 8,
    head_dim, 8]."""
    pages, heads, octets, page, eight = k_cache.shape
    assert eight == 8
    return _KV_CACHE.pack(pages, page, heads, octets * 8, _address(k_cache, _BF16, (pages, heads, octets, page, 8)),
                          _address(v_cache, _BF16, (pages, heads, page // 8, octets * 8, 8)))


def qblora_page_tables(context: torch.Tensor, fresh: torch.Tensor, page: int, free_pages: torch.Tensor, table: torch.Tensor,
                       tokens: int, starts: torch.Tensor = None, positions: torch.Tensor = None,
                       slots: torch.Tensor = None, taken: torch.Tensor = None):
    """Adds a step's pages to the block table (in place) and returns (starts, positions, slots, taken) of its new tokens;
    `tokens`: the room for them."""
    n, width = table.shape
    n_free = free_pages.shape[0]
    dev = table.device
    if starts is None and positions is None and taken is None:           # one allocation for the three of a type
        starts, positions, taken = torch.empty(n + tokens + 2, dtype=_I32, device=dev).split_with_sizes((n + 1, tokens, 1))
        p_starts = starts.data_ptr()
        p_positions, p_taken = p_starts + 4 * (n + 1), p_starts + 4 * (n + 1 + tokens)
    else:
        starts = torch.empty(n + 1, dtype=_I32, device=dev) if starts is None else starts
        positions = torch.empty(tokens, dtype=_I32, device=dev) if positions is None else positions
        taken = torch.empty(1, dtype=_I32, device=dev) if taken is None else taken
        p_starts, p_positions, p_taken = (_address(starts, _I32, (n + 1,)), _address(positions, _I32, (tokens,)),
                                          _address(taken, _I32, (1,)))
    if slots is None:
        slots = torch.empty(tokens, dtype=_I64, device=dev)
        p_slots = slots.data_ptr()
    else:
        p_slots = _address(slots, _I64, (tokens,))
    rc = lib().qblora_page_tables(_address(context, _I32, (n,)), _address(fresh, _I32, (n,)), n, page,
                                  _address(free_pages, _I32, (n_free,)), n_free, _address(table, _I32, (n, width)), width, tokens,
                                  p_starts, p_positions, p_slots, p_taken, _current_stream())
    if rc:
        _check(rc, "qblora_page_tables")
    return starts, positions, slots, taken


def qblora_rope_frequencies(rot: int, base: float = 10000.0, kind: int = ROPE_PLAIN, factor: float = 1.0,
                            original: float = 4096.0, low: float = 1.0, high: float = 32.0, device="cuda"):
    """(frequencies fp32 [rot / 2] on `device`, factor on q and k) for the scaling `kind` (ROPE_*)."""
    freq = np.empty(max(rot // 2, 0), np.float32)
    scale = C.c_float()
    rc = lib().qblora_rope_frequencies(rot, base, kind, factor, original, low, high, freq.ctypes.data_as(C.c_void_p),
                                       C.byref(scale))
    _check(rc, "qblora_rope_frequencies")
    return torch.from_numpy(freq).to(device), scale.value


def _rope(freq, interleaved, scale) -> bytes:
    half, = freq.shape
    return _ROPE.pack(2 * half, interleaved, scale, _address(freq, _F32, (half,)))


def _like(q, ld):
    """A contiguous array for the results of q, whose tokens are ld elements apart."""
    T, heads, dim = q.shape
    return torch.empty_like(q) if ld == heads * dim else torch.empty((T, heads, dim), dtype=_BF16, device=q.device)


def _rope_call(name, q, k, positions, freq, interleaved, scale, q_out, k_out):
    T, heads, dim = q.shape
    ldq, ld_out = _heads(q, T, heads, dim), heads * dim
    if q_out is None:
        q_out = _like(q, ldq)
    else:
        ld_out = _heads(q_out, T, heads, dim)
    if k is None:
        kv_heads = ldk = ldk_out = p_k = p_k_out = 0
        k_out = None
    else:
        kv_heads = k.shape[1]
        ldk, ldk_out = _heads(k, T, kv_heads, dim), kv_heads * dim
        if k_out is None:
            k_out = _like(k, ldk)
        else:
            ldk_out = _heads(k_out, T, kv_heads, dim)
        p_k, p_k_out = k.data_ptr(), k_out.data_ptr()
    rc = getattr(lib(), name)(_rope(freq, interleaved, scale), q.data_ptr(), ldq, heads, p_k, ldk, kv_heads, dim,
                              _address(positions, _I32, (T,)), T, q_out.data_ptr(), ld_out, p_k_out, ldk_out, _current_stream())
    if rc:
        _check(rc, name)
    return q_out, k_out


def qblora_rope_fwd(q: torch.Tensor, k, positions: torch.Tensor, freq: torch.Tensor, interleaved: bool = False,
                    scale: float = 1.0, q_out: torch.Tensor = None, k_out: torch.Tensor = None):
    """Rotary positions on q [T, heads, head_dim] and k [T, kv_heads, head_dim] (or None)."""
    return _rope_call("qblora_rope_fwd", q, k, positions, freq, interleaved, scale, q_out, k_out)


def qblora_rope_bwd(dq: torch.Tensor, dk, positions: torch.Tensor, freq: torch.Tensor, interleaved: bool = False,
                    scale: float = 1.0, dq_out: torch.Tensor = None, dk_out: torch.Tensor = None):
    """The gradients of q and k from those of the rotated ones."""
    return _rope_call("qblora_rope_bwd", dq, dk, positions, freq, interleaved, scale, dq_out, dk_out)


def qblora_rope_cache(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor,
                      freq: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, interleaved: bool = False,
                      scale: float = 1.0, q_out: torch.Tensor = None):
    """The rotated q; the rotated k and v go to their slots of the paged cache."""
    T, heads, dim = q.shape
    kv_heads = k_cache.shape[1]
    assert dim == 8 * k_cache.shape[2]
    ldq, ld_out = _heads(q, T, heads, dim), heads * dim
    if q_out is None:
        q_out = _like(q, ldq)
    else:
        ld_out = _heads(q_out, T, heads, dim)
    rc = lib().qblora_rope_cache(_rope(freq, interleaved, scale), q.data_ptr(), ldq, heads, k.data_ptr(),
                                 _heads(k, T, kv_heads, dim), v.data_ptr(), _heads(v, T, kv_heads, dim),
                                 _address(positions, _I32, (T,)), _address(slots, _I64, (T,)), T, q_out.data_ptr(), ld_out,
                                 _cache(k_cache, v_cache), _current_stream())
    if rc:
        _check(rc, "qblora_rope_cache")
    return q_out


def qblora_paged_attention_workspace_bytes(k_cache: torch.Tensor, v_cache: torch.Tensor, heads: int, max_new: int) -> int:
    return int(lib().qblora_paged_attention_workspace_bytes(_cache(k_cache, v_cache), heads, max_new))


def qblora_paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                           starts: torch.Tensor, context: torch.Tensor, scale: float, window: int = 0, max_new: int = None,
                           out: torch.Tensor = None, lse: torch.Tensor = None, workspace: torch.Tensor = None):
    """Attention of the new tokens q [T, heads, head_dim] of a batch over their requests' pages.  max_new: the most new
    tokens of a request, as far as it is known (default: T)."""
    T, heads, dim = q.shape
    n, width = table.shape
    assert dim == 8 * k_cache.shape[2]
    cache = _cache(k_cache, v_cache)
    ldq, ld_out = _heads(q, T, heads, dim), heads * dim
    if max_new is None:
        max_new = T
    dev = q.device
    if out is None:
        out = _like(q, ldq)
    else:
        ld_out = _heads(out, T, heads, dim)
    L = lib()
    if workspace is None:
        nbytes = L.qblora_paged_attention_workspace_bytes(cache, heads, max_new)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    rc = L.qblora_paged_attention(q.data_ptr(), ldq, heads, cache, _address(table, _I32, (n, width)), width,
                                  _address(starts, _I32, (n + 1,)), _address(context, _I32, (n,)), n, T, scale, window, max_new,
                                  out.data_ptr(), ld_out, None if lse is None else _address(lse, _F32, (T, heads)),
                                  workspace.data_ptr(), nbytes, _current_stream())
    if rc:
        _check(rc, "qblora_paged_attention")
    return out


def qblora_rms_norm_fwd(x: torch.Tensor, w: torch.Tensor, eps: float, residual: torch.Tensor = None, keep: bool = False,
                        total: torch.Tensor = None, y: torch.Tensor = None, rstd: torch.Tensor = None):
    """(y, total, rstd): the norm of total = x + residual (x itself without one); rstd, for the backward pass, is None unless
    `keep` is set or a tensor is given."""
    T, d = x.shape
    p_x, p_residual = _address(x, _BF16, (T, d)), None
    if y is None:
        y = torch.empty_like(x)
        p_y = y.data_ptr()
    else:
        p_y = _address(y, _BF16, (T, d))
    if residual is None:
        total, p_total = x, p_x
    else:
        p_residual = _address(residual, _BF16, (T, d))
        if total is None:
            total = torch.empty_like(x)
            p_total = total.data_ptr()
        else:
            p_total = _address(total, _BF16, (T, d))
    if keep and rstd is None:
        rstd = torch.empty(T, dtype=_F32, device=x.device)
    rc = lib().qblora_rms_norm_fwd(p_x, p_residual, _address(w, _BF16, (d,)), T, d, eps, p_total, p_y,
                                   None if rstd is None else _address(rstd, _F32, (T,)), _current_stream())
    if rc:
        _check(rc, "qblora_rms_norm_fwd")
    return y, total, rstd


def qblora_rms_norm_bwd_workspace_bytes(T: int, d: int) -> int:
    return int(lib().qblora_rms_norm_bwd_workspace_bytes(T, d))


def qblora_rms_norm_bwd(total: torch.Tensor, w: torch.Tensor, rstd: torch.Tensor, dy: torch.Tensor,
                        dtotal: torch.Tensor = None, need_dw: bool = True, dx: torch.Tensor = None, dw: torch.Tensor = None,
                        workspace: torch.Tensor = None):
    """(dx, dw): the gradients of the sum (x and residual alike) and of the weight."""
    T, d = total.shape
    dev = total.device
    p_total = _address(total, _BF16, (T, d))
    if dx is None:
        dx = torch.empty_like(total)
        p_dx = dx.data_ptr()
    else:
        p_dx = _address(dx, _BF16, (T, d))
    p_dw = p_ws = None
    nbytes = 0
    if need_dw:
        if dw is None:
            dw = torch.empty(d, dtype=_F32, device=dev)
            p_dw = dw.data_ptr()
        else:
            p_dw = _address(dw, _F32, (d,))
        if workspace is None:
            nbytes = lib().qblora_rms_norm_bwd_workspace_bytes(T, d)
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        else:
            nbytes = workspace.numel() * workspace.element_size()
        p_ws = workspace.data_ptr()
    rc = lib().qblora_rms_norm_bwd(p_total, _address(w, _BF16, (d,)), _address(rstd, _F32, (T,)), _address(dy, _BF16, (T, d)),
                                   None if dtotal is None else _address(dtotal, _BF16, (T, d)), T, d, p_dx,
                                   p_dw, p_ws, nbytes, _current_stream())
    if rc:
        _check(rc, "qblora_rms_norm_bwd")
    return dx, (dw if need_dw else None)


# ---- many adapters on one frozen projection -------------------------------------------------------------

def _current_device() -> int:
    return torch._C._cuda_getDevice()


def _here(*tensors) -> None:
    """The calls below launch on the current device: what they are given (None: nothing) has to lie there."""
    device = _current_device()
    for t in tensors:
        assert t is None or t.get_device() == device


class Adapters:
    """The adapters of one projection, by number, and the device table that describes them (qblora_adapter_table)."""

    def __init__(self, count, d_in, d_out, lambda1, lambda2, R, table):
        self.count, self.d_in, self.d_out, self.lambda1, self.lambda2, self.R = count, d_in, d_out, lambda1, lambda2, R
        self.table = table
        self.adapters, self.grads = [None] * count, [None] * count       # what the table points to stays alive

    def c_bytes(self) -> bytes:
        return _ADAPTERS.pack(self.count, self.d_in, self.d_out, self.lambda1, self.lambda2, self.R, self.table.data_ptr())


def qblora_adapter_table(adapters, d_in: int, d_out: int, lambda1: int = None, lambda2: int = None, R: int = None, grads=None,
                         device=None, into: Adapters = None, first: int = 0) -> Adapters:
    """The table of a list of Adapter (None: no adapter under that number).  R: room for adapters of higher ranks; grads: for
    each adapter the fp32 tensors (dA, dB) that qblora_adapters_bwd writes, or None.  `into`: writes them to an existing table
    instead, from number `first` on; the other entries stay."""
    some = next((a for a in adapters if a is not None and a.A is not None and a.B is not None), None)
    if into is None:
        lambda1 = some.lambda1 if lambda1 is None else lambda1
        lambda2 = some.lambda2 if lambda2 is None else lambda2
        R = max(a.R for a in adapters if a is not None) if R is None else R
        device = some.A.device if device is None else device
        count = first + len(adapters)
        table = torch.zeros(int(lib().qblora_adapter_table_bytes(count)), dtype=torch.uint8, device=device)
        into = Adapters(count, d_in, d_out, lambda1, lambda2, R, table)
    assert (into.d_in, into.d_out) == (d_in, d_out)
    _here(into.table)
    n = len(adapters)
    empty = Adapter(None, None, into.lambda1, into.lambda2, 0.0)
    for a in adapters:
        if a is not None and a.A is not None and a.B is not None:
            _here(a.A, a.B)
            _address(a.A, _BF16, (d_in // into.lambda1, a.R))
            _address(a.B, _BF16, (a.R, d_out // into.lambda2))
    pairs = [None] * n if grads is None else list(grads)
    assert len(pairs) == n
    for a, g in zip(adapters, pairs):
        if g is not None:
            _here(*g)
            _address(g[0], _F32, tuple(a.A.shape))
            _address(g[1], _F32, tuple(a.B.shape))
    raw = b"".join((empty if a is None else a).c_bytes() for a in adapters)
    dA, dB = ((C.c_void_p * n)(*[None if g is None else g[i].data_ptr() for g in pairs]) for i in (0, 1))
    _check(lib().qblora_adapter_table(into.c_bytes(), first, n, raw, dA, dB, _current_stream()), "qblora_adapter_table")
    into.adapters[first:first + n], into.grads[first:first + n] = list(adapters), pairs
    return into


def qblora_adapter_groups(starts: torch.Tensor, which: torch.Tensor, count: int, T: int, first: torch.Tensor = None,
                          order: torch.Tensor = None, tiles: torch.Tensor = None):
    """(first, order, tiles): the T tokens of a batch by adapter, which all projections share.  starts [n + 1], which [n]."""
    n, = which.shape
    _here(starts, which, first, order, tiles)
    L = lib()
    room = _tile_room(count, T)
    if first is None and order is None and tiles is None:                # one allocation; the tiles, which are 16 bytes each, lead it
        whole = torch.empty(4 * room + count + 1 + T, dtype=_I32, device=which.device)
        tiles, first, order = whole.split_with_sizes((4 * room, count + 1, T))
        p_tiles = whole.data_ptr()
        p_first, p_order, tiles = p_tiles + 16 * room, p_tiles + 16 * room + 4 * (count + 1), tiles.view(room, 4)
    else:
        first = torch.empty(count + 1, dtype=_I32, device=which.device) if first is None else first
        order = torch.empty(T, dtype=_I32, device=which.device) if order is None else order
        tiles = torch.empty((room, 4), dtype=_I32, device=which.device) if tiles is None else tiles
        p_first, p_order, p_tiles = (_address(first, _I32, (count + 1,)), _address(order, _I32, (T,)),
                                     _address(tiles, _I32, (room, 4)))
    rc = L.qblora_adapter_groups(_address(starts, _I32, (n + 1,)), _address(which, _I32, (n,)), n, count, T, p_first, p_order,
                                 p_tiles, _current_stream())
    if rc:
        _check(rc, "qblora_adapter_groups")
    return first, order, tiles


def _rows(t, T, width) -> int:
    """Elements from one row of a bf16 [T, width] to the next: any number, features one behind the other."""
    assert t.dtype is _BF16 and t.is_cuda and t.shape == (T, width)
    if t.is_contiguous():
        return width
    row, feature = t.stride()
    assert feature == 1 or width == 1
    return row if T > 1 else max(row, width)


def _tile_room(count, T) -> int:
    """qblora_adapter_tiles, without the call."""
    return -(-T // 64) + min(count, T)


def _groups(ads, groups, T):
    first, order, tiles = groups
    assert tiles.dim() == 2 and tiles.shape[0] == _tile_room(ads.count, T)
    return (_address(first, _I32, (ads.count + 1,)), _address(order, _I32, (T,)), _address(tiles, _I32, (tiles.shape[0], 4)))


def qblora_adapters_saved_bytes(ads: Adapters, T: int) -> int:
    return int(lib().qblora_adapters_saved_bytes(ads.c_bytes(), T))


def qblora_adapters_workspace_bytes(ads: Adapters, T: int) -> int:
    return int(lib().qblora_adapters_workspace_bytes(ads.c_bytes(), T))


def _saved(saved, L, a, T):
    if saved is None:
        return None
    assert saved.is_cuda and saved.is_contiguous() and saved.numel() * saved.element_size() >= L.qblora_adapters_saved_bytes(a, T)
    return saved.data_ptr()


def _adapters_workspace(workspace, L, a, T, device):
    if workspace is None:
        nbytes = L.qblora_adapters_workspace_bytes(a, T)
        return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes
    assert workspace.is_contiguous()
    return workspace, workspace.numel() * workspace.element_size()


def qblora_adapters_fwd(ads: Adapters, groups, X: torch.Tensor, Y: torch.Tensor, saved: torch.Tensor = None,
                        workspace: torch.Tensor = None):
    """Adds every token's adapter term to Y [T, d_out], in place.  groups: what qblora_adapter_groups returned."""
    T = X.shape[0]
    _here(X, Y, ads.table, *groups, saved, workspace)
    L, a = lib(), ads.c_bytes()
    ldx, ldy = _rows(X, T, ads.d_in), _rows(Y, T, ads.d_out)
    first, order, tiles = _groups(ads, groups, T)
    ws, nbytes = _adapters_workspace(workspace, L, a, T, X.device)
    rc = L.qblora_adapters_fwd(a, first, order, tiles, X.data_ptr(), ldx, T, Y.data_ptr(), ldy, _saved(saved, L, a, T),
                               ws.data_ptr(), nbytes, _current_stream())
    if rc:
        _check(rc, "qblora_adapters_fwd")
    return Y


def qblora_adapters_bwd(ads: Adapters, groups, X, dY: torch.Tensor, dX: torch.Tensor = None, gradients: bool = True,
                        saved: torch.Tensor = None, workspace: torch.Tensor = None):
    """Adds the adapters' part to dX [T, d_in] (if given), in place, and writes the gradients of the table's adapters.  X may be
    None without gradients; saved: what the forward call filled."""
    T = dY.shape[0]
    _here(X, dY, dX, ads.table, *groups, saved, workspace)
    L, a = lib(), ads.c_bytes()
    ldx = 0 if X is None else _rows(X, T, ads.d_in)
    lddx = 0 if dX is None else _rows(dX, T, ads.d_in)
    lddy = _rows(dY, T, ads.d_out)
    first, order, tiles = _groups(ads, groups, T)
    ws, nbytes = _adapters_workspace(workspace, L, a, T, dY.device)
    rc = L.qblora_adapters_bwd(a, first, order, tiles, _ptr(X), ldx, dY.data_ptr(), lddy, T, _saved(saved, L, a, T), _ptr(dX),
                               lddx, gradients, ws.data_ptr(), nbytes, _current_stream())
    if rc:
        _check(rc, "qblora_adapters_bwd")
    return dX


# ---- the optimizer's step -------------------------------------------------------------------------------

class AdamWList:
    """The tensors of a step: the C struct, and everything its device plan points to."""

    def __init__(self, c, plan, tensors):
        self.c, self.plan, self.tensors = c, plan, tensors
        self.raw = bytes(c)
        self.norm_bytes = int(lib().qblora_grad_norm_workspace_bytes(self.raw))


def qblora_adamw_list(params, grads, m, v, master=None, m_scale=None, v_scale=None, rate=1.0, decay=0.0) -> AdamWList:
    """One list of tensors for qblora_grad_norm and qblora_adamw_step, each argument a list with an entry for each tensor:
    params bf16 (entries may be None where there is a master), grads fp32, moments m and v fp32, or float8_e4m3fn and float8_e5m2
    with their scales; master fp32 or None; rate and decay: numbers for all, or a list."""
    n = len(grads)
    each = lambda x: list(x) if isinstance(x, (list, tuple)) else [x] * n  # noqa: E731
    params, master, m_scale, v_scale, rate, decay = (each(x) for x in (params, master, m_scale, v_scale, rate, decay))
    bits = 8 if n and m[0].dtype is torch.float8_e4m3fn else 32
    types = (torch.float8_e4m3fn, torch.float8_e5m2) if bits == 8 else (_F32, _F32)
    assert all(len(x) == n for x in (params, m, v, master, m_scale, v_scale, rate, decay))
    _here(*params, *grads, *m, *v, *master, *m_scale, *v_scale)
    c = (CAdamWTensor * max(n, 1))()
    for i in range(n):
        shape = grads[i].shape
        k = grads[i].numel()
        blocks = (-(-k // 256),)
        c[i] = CAdamWTensor(k, None if params[i] is None else _address(params[i], _BF16, shape),
                            None if master[i] is None else _address(master[i], _F32, shape), _address(grads[i], _F32, shape),
                            _address(m[i], types[0], shape), _address(v[i], types[1], shape),
                            _address(m_scale[i], _F32, blocks) if bits == 8 else None,
                            _address(v_scale[i], _F32, blocks) if bits == 8 else None, rate[i], decay[i])
    plan = torch.empty(int(lib().qblora_adamw_plan_bytes(c, n)), dtype=torch.uint8,
                       device=grads[0].device if n else "cuda")
    out = CAdamWList()
    _check(lib().qblora_adamw_plan(c, n, bits, plan.data_ptr() or None, plan.numel(), C.byref(out), _current_stream()),
           "qblora_adamw_plan")
    return AdamWList(out, plan, (params, list(grads), list(m), list(v), master, m_scale, v_scale))


def qblora_grad_norm(tensors: AdamWList, max_norm: float, out: torch.Tensor = None, workspace: torch.Tensor = None):
    """fp32 [2] on the device: the norm of all gradients, and the factor that clips it to max_norm."""
    dev = tensors.plan.device
    _here(tensors.plan, out, workspace)
    if out is None:
        out = torch.empty(2, dtype=_F32, device=dev)
    if workspace is None:
        workspace = torch.empty(tensors.norm_bytes, dtype=torch.uint8, device=dev)
    assert workspace.is_contiguous()
    rc = lib().qblora_grad_norm(tensors.raw, max_norm, _address(out, _F32, (2,)), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _current_stream())
    if rc:
        _check(rc, "qblora_grad_norm")
    return out


def qblora_adamw_step(tensors: AdamWList, step, lr, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                      clip: torch.Tensor = None, seed: int = 0) -> None:
    """One AdamW step on every tensor of the list, in place.  step, lr: numbers, or one-element tensors on the device (int64 and
    fp32) that the call reads when it runs, as a captured graph needs; clip: what qblora_grad_norm returned."""
    p_step = p_lr = 0
    _here(tensors.plan, clip)
    if isinstance(step, torch.Tensor):
        _here(step)
        assert step.numel() == 1
        step, p_step = 1, _address(step, _I64, step.shape)
    if isinstance(lr, torch.Tensor):
        _here(lr)
        assert lr.numel() == 1
        lr, p_lr = 0.0, _address(lr, _F32, lr.shape)
    how = _ADAMW.pack(lr, beta1, beta2, eps, step, p_step, p_lr, seed & 0xffffffff)
    rc = lib().qblora_adamw_step(tensors.raw, how, None if clip is None else _address(clip, _F32, (2,)), _current_stream())
    if rc:
        _check(rc, "qblora_adamw_step")
