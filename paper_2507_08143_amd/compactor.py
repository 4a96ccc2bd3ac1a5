"""Thin ctypes binding of libcompactor.so (argument marshalling only).

Every function here has the name of the C entry point it calls
(include/compactor.h; those of the cache in 4 bits a second one) and does
nothing but turn torch tensors into raw device pointers, allocate the outputs
with torch, and check the return code.  All of
the method's arithmetic runs in the HIP kernels; there is no CPU fallback: if
the shared library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("COMPACTOR_LIB", os.path.join(_HERE, "libcompactor.so"))

if not os.path.exists(_LIB_PATH):
    raise ImportError(
        "libcompactor.so is not built: run `python -m paper_2507_08143_amd.build` "
        "(needs hipcc; cross-compiles for gfx950 without a GPU)")

_lib = C.CDLL(_LIB_PATH)

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EALIGN, EHIP = 0, -1, -2, -3, -4, -5
STATUS_OK, STATUS_PIVOT, STATUS_NONFINITE = 0, 1, 2


class _Request(C.Structure):
    _fields_ = [("k_score", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("attn", C.c_void_p), ("stride_l", C.c_int64), ("stride_h", C.c_int64),
                ("stride_t", C.c_int64), ("n", C.c_int32), ("ratio", C.c_float)]


class _Params(C.Structure):
    _fields_ = [("layers", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("sketch_dim", C.c_int32), ("phi", C.c_void_p), ("ridge_rel", C.c_float),
                ("lambda_blend", C.c_float), ("group_bytes", C.c_int64),
                ("gram_wgs", C.c_int32), ("score_tokens", C.c_int32),
                ("select_scope", C.c_int32), ("stage_events", C.c_void_p)]


class _AttnRequest(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p),
                ("q_stride_l", C.c_int64), ("q_stride_h", C.c_int64), ("q_stride_t", C.c_int64),
                ("k_stride_l", C.c_int64), ("k_stride_h", C.c_int64), ("k_stride_t", C.c_int64),
                ("n", C.c_int32)]


class _AttnParams(C.Structure):
    _fields_ = [("layers", C.c_int32), ("kv_heads", C.c_int32), ("q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("chunk", C.c_int32), ("pool", C.c_int32),
                ("scale", C.c_float)]


class _PagePool(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("page_stride", C.c_int64), ("layer_stride", C.c_int64),
                ("head_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("page_size", C.c_int32), ("num_pages", C.c_int32)]


class _PageTable(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("len", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("pool", _PagePool), ("tables", C.c_void_p), ("table_stride", C.c_int64),
                ("table_len", C.c_int32), ("nreq", C.c_int32), ("layers", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("counts", C.c_void_p),
                ("seen", C.c_void_p), ("count_stride_b", C.c_int64), ("count_stride_l", C.c_int64),
                ("mass", C.c_void_p), ("positions", C.c_void_p), ("state_page_stride", C.c_int64),
                ("state_layer_stride", C.c_int64), ("state_head_stride", C.c_int64)]


class _CacheRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride_b", C.c_int64), ("stride_l", C.c_int64),
                ("stride_t", C.c_int64), ("stride_h", C.c_int64), ("new_tokens", C.c_void_p),
                ("tokens", C.c_int32)]


class _CacheQuery(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("q_stride_b", C.c_int64), ("q_stride_l", C.c_int64), ("q_stride_t", C.c_int64),
                ("q_stride_h", C.c_int64), ("out_stride_b", C.c_int64), ("out_stride_l", C.c_int64),
                ("out_stride_t", C.c_int64), ("out_stride_h", C.c_int64), ("new_tokens", C.c_void_p),
                ("tokens", C.c_int32), ("q_heads", C.c_int32), ("scale", C.c_float),
                ("softcap", C.c_float), ("accumulate", C.c_int32), ("max_tokens", C.c_int32)]


class _CacheEvict(C.Structure):
    _fields_ = [("budget", C.c_int32), ("budgets", C.c_void_p), ("sink", C.c_int32),
                ("recent", C.c_int32), ("scope", C.c_int32), ("max_tokens", C.c_int32)]


class _MxCache(C.Structure):
    _fields_ = [("cache", _Cache), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p)]


class _CacheRowsOut(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride_b", C.c_int64), ("stride_l", C.c_int64),
                ("stride_t", C.c_int64), ("stride_h", C.c_int64), ("new_tokens", C.c_void_p),
                ("tokens", C.c_int32), ("first", C.c_int32)]


class _Rotation(C.Structure):
    _fields_ = [("freqs", C.c_void_p), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32),
                ("q_norm", C.c_void_p), ("k_norm", C.c_void_p), ("eps", C.c_float)]


class _RotateRows(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "q_out", "k_out", "k_plain")] +
                [("%s_stride_%s" % (n, d), C.c_int64) for n in ("q", "k", "q_out", "k_out", "k_plain") for d in "blth"] +
                [("positions", C.c_void_p), ("position_stride_b", C.c_int64), ("new_tokens", C.c_void_p)] +
                [(n, C.c_int32) for n in ("nreq", "layers", "tokens", "q_heads", "kv_heads")])


class _RotateQueries(C.Structure):
    _fields_ = ([("q", C.c_void_p), ("q_out", C.c_void_p)] +
                [("%s_stride_%s" % (n, d), C.c_int64) for n in ("q", "q_out") for d in "blth"] + [("q_heads", C.c_int32)])


class _PagesReserve(C.Structure):
    _fields_ = [("refs", C.c_void_p), ("new_tokens", C.c_void_p), ("tokens", C.c_int32), ("own_all", C.c_int32),
                ("pairs", C.c_void_p), ("done", C.c_void_p)]


_PP, _RP = C.POINTER(_Params), C.POINTER(_Request)
_CP, _CQP, _CEP = C.POINTER(_Cache), C.POINTER(_CacheQuery), C.POINTER(_CacheEvict)
_lib.compactor_cache_admit.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, _CP,
                                       C.c_void_p]
_lib.compactor_cache_append.argtypes = [_CP, C.POINTER(_CacheRows), C.c_void_p]
_lib.compactor_cache_attention.argtypes = [_CP, _CQP, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_cache_attention_workspace_size.argtypes = [_CP, _CQP, C.POINTER(C.c_size_t)]
_lib.compactor_cache_evict.argtypes = [_CP, _CEP, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_cache_evict_workspace_size.argtypes = [_CP, _CEP, C.POINTER(C.c_size_t)]
_MXP = C.POINTER(_MxCache)
_lib.compactor_mx_append.argtypes = [_MXP, C.POINTER(_CacheRows), C.c_void_p]
_lib.compactor_mx_store.argtypes = [_MXP, _CP, C.c_void_p]
_lib.compactor_mx_read.argtypes = [_MXP, C.POINTER(_CacheRowsOut), C.c_void_p]
_lib.compactor_mx_attention.argtypes = [_MXP, _CQP, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_mx_attention_workspace_size.argtypes = [_MXP, _CQP, C.POINTER(C.c_size_t)]
_lib.compactor_mx_evict.argtypes = [_MXP, _CEP, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_mx_evict_workspace_size.argtypes = [_MXP, _CEP, C.POINTER(C.c_size_t)]
_ROP = C.POINTER(_Rotation)
_lib.compactor_rotate.argtypes = [_ROP, C.POINTER(_RotateRows), C.c_void_p]
_lib.compactor_cache_append_rotated.argtypes = [_CP, _ROP, C.POINTER(_CacheRows), C.POINTER(_RotateQueries), C.c_void_p]
_lib.compactor_mx_append_rotated.argtypes = [_MXP, _ROP, C.POINTER(_CacheRows), C.POINTER(_RotateQueries), C.c_void_p]
_lib.compactor_pages_reserve.argtypes = [_CP, C.POINTER(_PagesReserve), C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_pages_reserve_workspace_size.argtypes = [_CP, C.POINTER(C.c_size_t)]
_lib.compactor_pages_compact_workspace_size.argtypes = [_CP, C.POINTER(C.c_size_t)]
_lib.compactor_pages_copy.argtypes = [_CP, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
_lib.compactor_mx_pages_copy.argtypes = [_MXP, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
_lib.compactor_pages_fork.argtypes = [_CP, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.compactor_pages_release.argtypes = [_CP, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.compactor_pages_compact.argtypes = [_CP, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
_APP, _ARP = C.POINTER(_AttnParams), C.POINTER(_AttnRequest)
_lib.compactor_attention_workspace_size.argtypes = [_APP, _ARP, C.c_int32, C.POINTER(C.c_size_t)]
_lib.compactor_attention_scores.argtypes = [_APP, _ARP, C.c_int32, C.c_void_p, C.c_void_p,
                                            C.c_size_t, C.c_void_p]
_lib.compactor_default_params.argtypes = [_PP, C.c_int32, C.c_int32]
_lib.compactor_default_params.restype = None
_lib.compactor_keep_count.argtypes = [C.c_int32, C.c_float]
_lib.compactor_keep_count.restype = C.c_int32
_lib.compactor_layout.argtypes = [_PP, _RP, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                  C.POINTER(C.c_int32)]
_lib.compactor_srht_phi.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.compactor_workspace_size.argtypes = [_PP, _RP, C.c_int32, C.POINTER(C.c_size_t)]
_lib.compactor_score.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_size_t, C.c_void_p]
_lib.compactor_select.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_size_t, C.c_void_p]
_lib.compactor_compact.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p]
_lib.compactor_compact_paged.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p,
                                         C.POINTER(_PagePool), C.POINTER(_PageTable), C.c_int32,
                                         C.c_void_p]
_lib.compactor_compress.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                    C.c_void_p]
_lib.compactor_compress_static.argtypes = [_PP, _RP, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.compactor_calibrated_ratio.argtypes = [C.c_double] * 4
_lib.compactor_calibrated_ratio.restype = C.c_double
_lib.compactor_error_string.argtypes = [C.c_int]
_lib.compactor_error_string.restype = C.c_char_p
_lib.compactor_version.restype = C.c_char_p

EXPORTS = ["compactor_default_params", "compactor_keep_count", "compactor_layout",
           "compactor_workspace_size", "compactor_srht_phi", "compactor_score", "compactor_select",
           "compactor_compact", "compactor_compact_paged", "compactor_compress", "compactor_compress_static",
           "compactor_calibrated_ratio",
           "compactor_error_string", "compactor_version",
           "compactor_attention_workspace_size", "compactor_attention_scores",
           "compactor_cache_admit", "compactor_cache_append", "compactor_cache_attention",
           "compactor_cache_attention_workspace_size", "compactor_cache_evict",
           "compactor_cache_evict_workspace_size",
           "compactor_mx_append", "compactor_mx_store", "compactor_mx_read", "compactor_mx_attention",
           "compactor_mx_attention_workspace_size", "compactor_mx_evict", "compactor_mx_evict_workspace_size",
           "compactor_rotate", "compactor_cache_append_rotated", "compactor_mx_append_rotated",
           "compactor_pages_reserve", "compactor_pages_reserve_workspace_size", "compactor_pages_compact",
           "compactor_pages_compact_workspace_size", "compactor_pages_copy", "compactor_mx_pages_copy",
           "compactor_pages_fork", "compactor_pages_release"]


STAGES = ["gram", "reduce", "solve", "score", "blend", "select", "gather"]


class StageEvents:
    """COMPACTOR_NUM_STAGES+1 raw hipEvent_t for compactor_params_t.stage_events, created
    through the HIP runtime that torch has already loaded."""

    def __init__(self):
        self._hip = C.CDLL("libamdhip64.so")
        self._hip.hipEventCreate.argtypes = [C.POINTER(C.c_void_p)]
        self._hip.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        self._hip.hipEventDestroy.argtypes = [C.c_void_p]
        self.array = (C.c_void_p * (len(STAGES) + 1))()
        for i in range(len(STAGES) + 1):
            ev = C.c_void_p()
            if self._hip.hipEventCreate(C.byref(ev)) != 0:
                raise RuntimeError("hipEventCreate failed")
            self.array[i] = ev

    def elapsed_ms(self):
        """-> {stage: ms} for the stages whose two events were recorded (after a stream sync)."""
        out = {}
        for i, name in enumerate(STAGES):
            ms = C.c_float(0)
            if self._hip.hipEventElapsedTime(C.byref(ms), self.array[i], self.array[i + 1]) == 0:
                out[name] = float(ms.value)
        self._hip.hipGetLastError()     # asking about a stage that did not run leaves an error pending
        return out

    def __del__(self):
        try:
            for ev in self.array:
                if ev:
                    self._hip.hipEventDestroy(ev)
        except Exception:
            pass


class CompactorError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__("libcompactor: %s (%d)" % (compactor_error_string(code), code))


def _check(rc: int):
    if rc != OK:
        raise CompactorError(rc)


def _refuse(what: str):
    raise ValueError("compactor: " + what)


def _require(cond: bool, what: str):
    """The C boundary takes plain pointers and cannot see a tensor's size, type or device: what it
    cannot check is checked here, before anything reaches the GPU.  (Checks whose message has to be
    put together test first and call _refuse: a call makes dozens of them.)"""
    if not cond:
        _refuse(what)


def _out(t: Optional[torch.Tensor], numel: int, dtype, name: str):
    """A caller-supplied output (or flat input) buffer: right type, dense, large enough, on the GPU."""
    if t is None:
        return
    if t.dtype != dtype:
        _refuse("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        _refuse("%s must be contiguous" % name)
    if t.numel() < numel:
        _refuse("%s holds %d elements, %d needed" % (name, t.numel(), numel))
    if not t.is_cuda:
        _refuse("%s must live on the GPU" % name)


def _int32(**values):
    """A number that the C structures would cut to its last 32 bits."""
    for name, x in values.items():
        if not 0 <= x < 1 << 31:
            _refuse("%s must be one of 0 .. 2^31 - 1, got %s" % (name, x))


SCOPE_HEAD, SCOPE_LAYER = 0, 1


@dataclass
class Params:
    layers: int
    kv_heads: int
    sketch_dim: int = 48
    phi: Optional[torch.Tensor] = None        # fp32 [128, sketch_dim] on the device
    ridge_rel: float = 0.0
    lambda_blend: float = 0.3
    group_bytes: int = 0
    head_dim: int = 128
    stage_events: Optional["StageEvents"] = None   # profiling aid (see the header)
    gram_wgs: int = 0                              # tuning knobs, 0 = library's choice
    score_tokens: int = 0
    select_scope: int = 0                           # SCOPE_HEAD, or SCOPE_LAYER (head-adaptive)

    def check_gpu(self):
        if self.phi is not None and self.sketch_dim > 0:
            _require(self.phi.is_cuda, "phi must live on the GPU")

    def c(self, on_gpu: bool = True) -> _Params:
        phi = 0
        if self.phi is not None and self.sketch_dim > 0:
            _require(self.phi.dtype == torch.float32 and self.phi.is_contiguous(),
                     "phi must be a contiguous float32 tensor")
            if tuple(self.phi.shape) != (self.head_dim, self.sketch_dim):
                _refuse("phi must have shape [head_dim, sketch_dim] = [%d, %d], got %s"
                        % (self.head_dim, self.sketch_dim, tuple(self.phi.shape)))
            if on_gpu:
                self.check_gpu()
            phi = self.phi.data_ptr()
        ev = C.cast(self.stage_events.array, C.c_void_p) if self.stage_events is not None else None
        return _Params(self.layers, self.kv_heads, self.head_dim, self.sketch_dim, phi,
                       self.ridge_rel, self.lambda_blend, self.group_bytes, self.gram_wgs,
                       self.score_tokens, self.select_scope, ev)


@dataclass
class Request:
    k_score: torch.Tensor                      # bf16 [L, H, n, d], d contiguous
    v_cache: torch.Tensor                      # bf16, same shape and strides
    ratio: float
    k_cache: Optional[torch.Tensor] = None     # bf16, same shape and strides; None = k_score
    attn: Optional[torch.Tensor] = None        # fp32 [L, H, n] contiguous

    def check_gpu(self):
        for name, t in (("v_cache", self.v_cache), ("k_cache", self.k_cache), ("attn", self.attn),
                        ("k_score", self.k_score)):
            if t is not None and not t.is_cuda:
                _refuse("%s must live on the GPU" % name)

    def c(self, params: Optional["Params"] = None, on_gpu: bool = True) -> _Request:
        k = self.k_score
        _require(k.dtype == torch.bfloat16 and k.dim() == 4 and k.stride(3) == 1,
                 "k_score must be a bfloat16 tensor [L, H, n, d] with d contiguous")
        shape, stride = k.shape, k.stride()
        if params is not None and not (shape[0] == params.layers and shape[1] == params.kv_heads and
                                       shape[3] == params.head_dim):
            _refuse("k_score has shape %s, the parameters say [%d, %d, n, %d]"
                    % (tuple(shape), params.layers, params.kv_heads, params.head_dim))
        for name, t in (("v_cache", self.v_cache), ("k_cache", self.k_cache)):
            if t is not None and t is not k:
                if t.dtype != torch.bfloat16 or t.shape != shape or t.stride() != stride:
                    _refuse("%s must be bfloat16 with the shape and strides of k_score" % name)
        if self.attn is not None:
            _require(self.attn.dtype == torch.float32 and self.attn.is_contiguous() and
                     self.attn.numel() >= shape[0] * shape[1] * shape[2],
                     "attn must be a contiguous float32 tensor of L*H*n elements")
        if on_gpu:
            self.check_gpu()
        return _Request(k.data_ptr(),
                        self.k_cache.data_ptr() if self.k_cache is not None else 0,
                        self.v_cache.data_ptr() if self.v_cache is not None else 0,
                        self.attn.data_ptr() if self.attn is not None else 0,
                        stride[0], stride[1], stride[2], shape[2], self.ratio)


def _marshal(params: Params, reqs: Sequence[Request], on_gpu: bool = True):
    _require(len(reqs) >= 1, "at least one request is needed")
    arr = (_Request * len(reqs))(*[r.c(params, on_gpu) for r in reqs])
    return C.byref(params.c(on_gpu)), arr, len(reqs)


def _check_gpu(params: Params, reqs: Sequence[Request]):
    """The part of the marshalling that asks where the tensors live.  The entry points marshal once,
    without it, to learn the sizes, and come back to this before the call."""
    for r in reqs:
        r.check_gpu()
    params.check_gpu()


def _ptr(t: Optional[torch.Tensor]):
    return 0 if t is None else t.data_ptr()


# the current stream's handle without the Stream object that torch.cuda.current_stream() builds (3 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return C.c_void_p(_raw_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _empty(stream, *shape, returned=True, **kw):
    """torch.empty for a call on `stream` (None: the current one).  The block comes from the pool of that stream: one of the current
    stream's pool may still be in use there by work that was enqueued before and has given it back.  returned: the caller gets
    the tensor, so the block waits for the caller's stream too when it is given back."""
    return _made_on(stream, lambda: torch.empty(*shape, **kw), returned)


def _made_on(stream, make, returned=True):
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        t = make()
    if returned and t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _device(reqs):
    return reqs[0].k_score.device


def compactor_version() -> str:
    return _lib.compactor_version().decode()


def compactor_error_string(code: int) -> str:
    return _lib.compactor_error_string(code).decode()


def compactor_keep_count(n: int, ratio: float) -> int:
    return int(_lib.compactor_keep_count(n, ratio))


def compactor_calibrated_ratio(nll: float, alpha: float, beta: float, tau: float) -> float:
    return float(_lib.compactor_calibrated_ratio(nll, alpha, beta, tau))


def compactor_default_params(layers: int, kv_heads: int) -> Params:
    p = _Params()
    _lib.compactor_default_params(C.byref(p), layers, kv_heads)
    return Params(p.layers, p.kv_heads, p.sketch_dim, None, p.ridge_rel, p.lambda_blend,
                  p.group_bytes, p.head_dim, None, p.gram_wgs, p.score_tokens, p.select_scope)


def compactor_srht_phi(sketch_dim: int, signs, cols, device, stream=None) -> torch.Tensor:
    """SRHT right-sketch (App. D) -> fp32 [128, sketch_dim] on `device`.  signs: 128 values
    (nonzero = -1); cols: sketch_dim distinct rows of the Hadamard matrix."""
    sg = (C.c_uint8 * 128)(*[1 if int(x) else 0 for x in signs])
    cl = (C.c_int32 * len(cols))(*[int(x) for x in cols])
    _require(len(signs) == 128 and len(cols) == sketch_dim,
             "signs must hold 128 values and cols sketch_dim values")
    phi = _empty(stream, 128, sketch_dim, dtype=torch.float32, device=device)
    with torch.cuda.device(phi.device):
        _check(_lib.compactor_srht_phi(sketch_dim, sg, cl, _ptr(phi), _stream(stream)))
    return phi


def _layout(pp, arr, n):
    so, ko, kk = (C.c_int64 * (n + 1))(), (C.c_int64 * (n + 1))(), (C.c_int32 * n)()
    _check(_lib.compactor_layout(pp, arr, n, so, ko, kk))
    return list(so), list(ko), list(kk)


def compactor_layout(params: Params, reqs: Sequence[Request]):
    """-> (score_off[nreq+1], kept_off[nreq+1], k_keep[nreq]) as Python lists."""
    return _layout(*_marshal(params, reqs, on_gpu=False))      # a host helper: sizes only


def _workspace_bytes(pp, arr, n) -> int:
    out = C.c_size_t(0)
    _check(_lib.compactor_workspace_size(pp, arr, n, C.byref(out)))
    return int(out.value)


def compactor_workspace_size(params: Params, reqs: Sequence[Request]) -> int:
    return _workspace_bytes(*_marshal(params, reqs, on_gpu=False))


def _workspace(call, reqs, workspace, stream=None):
    if workspace is None:
        nbytes = max(256, _workspace_bytes(*call))
        workspace = _empty(stream, nbytes, dtype=torch.uint8, device=_device(reqs))
    return workspace


def compactor_score(params: Params, reqs: Sequence[Request], scores=None, status=None,
                    workspace=None, stream=None):
    """-> (scores fp32 [sum L*H*n], status int32 [nreq*L*H])"""
    pp, arr, n = call = _marshal(params, reqs, on_gpu=False)
    so, _, _ = _layout(*call)
    dev, nh = _device(reqs), n * params.layers * params.kv_heads
    given = scores, status, workspace          # what is allocated here needs no check
    if scores is None:
        scores = _empty(stream, so[-1], dtype=torch.float32, device=dev)
    if status is None:
        status = _empty(stream, nh, dtype=torch.int32, device=dev)
    workspace = _workspace(call, reqs, workspace, stream)
    _check_gpu(params, reqs)
    _out(given[0], so[-1], torch.float32, "scores")
    _out(given[1], nh, torch.int32, "status")
    _out(given[2], 0, torch.uint8, "workspace")
    _check(_lib.compactor_score(pp, arr, n, _ptr(scores), _ptr(status), _ptr(workspace),
                                workspace.numel(), _stream(stream)))
    return scores, status


def compactor_select(params: Params, reqs: Sequence[Request], scores: torch.Tensor,
                     kept_idx=None, kept_cnt=None, workspace=None, stream=None):
    """-> (kept_idx int32 [sum L*H*k_keep], kept_cnt int32 [nreq*L*H])"""
    pp, arr, n = call = _marshal(params, reqs, on_gpu=False)
    so, ko, _ = _layout(*call)
    dev, nh = scores.device, n * params.layers * params.kv_heads
    if kept_idx is None:
        kept_idx = _empty(stream, ko[-1], dtype=torch.int32, device=dev)
    if kept_cnt is None:
        kept_cnt = _empty(stream, nh, dtype=torch.int32, device=dev)
    _check_gpu(params, reqs)
    workspace = _workspace(call, reqs, workspace, stream)
    _out(scores, so[-1], torch.float32, "scores")       # the scores' device decides where the others live
    _out(kept_idx, ko[-1], torch.int32, "kept_idx")
    _out(kept_cnt, nh, torch.int32, "kept_cnt")
    _out(workspace, 0, torch.uint8, "workspace")
    _check(_lib.compactor_select(pp, arr, n, _ptr(scores), _ptr(kept_idx), _ptr(kept_cnt),
                                 _ptr(workspace), workspace.numel(), _stream(stream)))
    return kept_idx, kept_cnt


def compactor_compact(params: Params, reqs: Sequence[Request], kept_idx: torch.Tensor,
                      kept_cnt: torch.Tensor, k_packed=None, v_packed=None, stream=None):
    """-> (k_packed, v_packed) bf16 [sum L*H*k_keep, d]"""
    pp, arr, n = call = _marshal(params, reqs, on_gpu=False)
    _, ko, _ = _layout(*call)
    dev = _device(reqs)
    if k_packed is None:
        k_packed = _empty(stream, ko[-1], params.head_dim, dtype=torch.bfloat16, device=dev)
    if v_packed is None:
        v_packed = _empty(stream, ko[-1], params.head_dim, dtype=torch.bfloat16, device=dev)
    _check_gpu(params, reqs)
    _out(kept_idx, ko[-1], torch.int32, "kept_idx")
    _out(kept_cnt, n * params.layers * params.kv_heads, torch.int32, "kept_cnt")
    _out(k_packed, ko[-1] * params.head_dim, torch.bfloat16, "k_packed")
    _out(v_packed, ko[-1] * params.head_dim, torch.bfloat16, "v_packed")
    _check(_lib.compactor_compact(pp, arr, n, _ptr(kept_idx), _ptr(kept_cnt), _ptr(k_packed),
                                  _ptr(v_packed), _stream(stream)))
    return k_packed, v_packed


def compactor_compact_paged(params: Params, reqs: Sequence[Request], kept_idx: torch.Tensor,
                            kept_cnt: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                            tables: Sequence[torch.Tensor], in_place: bool = False, stream=None):
    """Retained rows into a paged cache.  k_pages / v_pages: bf16 views indexed
    [page, layer, slot, head, channel] (any strides, channel contiguous, the same for both);
    tables[b]: int32 device tensor, physical page of each logical page of request b."""
    _require(k_pages.dtype == torch.bfloat16 and v_pages.dtype == torch.bfloat16,
             "k_pages and v_pages must be bfloat16")
    _require(k_pages.dim() == 5 and k_pages.stride(4) == 1 and v_pages.shape == k_pages.shape and
             v_pages.stride() == k_pages.stride(),
             "k_pages and v_pages must be [page, layer, slot, head, channel] views of equal shape and "
             "strides, channel contiguous")
    _require(k_pages.shape[1] == params.layers and k_pages.shape[3] == params.kv_heads and
             k_pages.shape[4] == params.head_dim,
             "the page pool has shape %s, the parameters say [pages, %d, slots, %d, %d]"
             % (tuple(k_pages.shape), params.layers, params.kv_heads, params.head_dim))
    _require(k_pages.is_cuda and v_pages.is_cuda, "the page pool must live on the GPU")
    pool = _PagePool(k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1),
                     k_pages.stride(3), k_pages.stride(2), k_pages.shape[2], k_pages.shape[0])
    for t in tables:
        _out(t, 0, torch.int32, "a block table")
    tabs = (_PageTable * len(tables))(*[_PageTable(t.data_ptr(), t.numel()) for t in tables])
    pp, arr, n = call = _marshal(params, reqs)
    _require(len(tables) == n, "one block table per request is needed")
    _, ko, _ = _layout(*call)
    _out(kept_idx, ko[-1], torch.int32, "kept_idx")
    _out(kept_cnt, n * params.layers * params.kv_heads, torch.int32, "kept_cnt")
    _check(_lib.compactor_compact_paged(pp, arr, n, _ptr(kept_idx), _ptr(kept_cnt), C.byref(pool),
                                        tabs, 1 if in_place else 0, _stream(stream)))


def compactor_compress(params: Params, reqs: Sequence[Request], want_scores: bool = False,
                       scores=None, kept_idx=None, kept_cnt=None, k_packed=None, v_packed=None,
                       status=None, workspace=None, stream=None):
    """Fused score -> select -> compact.  -> dict of the output tensors."""
    pp, arr, n = call = _marshal(params, reqs, on_gpu=False)
    so, ko, _ = _layout(*call)
    dev = _device(reqs)
    nh = n * params.layers * params.kv_heads
    # what is allocated here needs no check
    given = scores, kept_idx, kept_cnt, k_packed, v_packed, status, workspace
    if scores is None and want_scores:
        scores = _empty(stream, so[-1], dtype=torch.float32, device=dev)
    if kept_idx is None:
        kept_idx = _empty(stream, ko[-1], dtype=torch.int32, device=dev)
    if kept_cnt is None:
        kept_cnt = _empty(stream, nh, dtype=torch.int32, device=dev)
    if k_packed is None:
        k_packed = _empty(stream, ko[-1], params.head_dim, dtype=torch.bfloat16, device=dev)
    if v_packed is None:
        v_packed = _empty(stream, ko[-1], params.head_dim, dtype=torch.bfloat16, device=dev)
    if status is None:
        status = _empty(stream, nh, dtype=torch.int32, device=dev)
    workspace = _workspace(call, reqs, workspace, stream)
    _check_gpu(params, reqs)
    for t, numel, dtype, name in zip(
            given, (so[-1], ko[-1], nh, ko[-1] * params.head_dim, ko[-1] * params.head_dim, nh, 0),
            (torch.float32, torch.int32, torch.int32, torch.bfloat16, torch.bfloat16, torch.int32, torch.uint8),
            ("scores", "kept_idx", "kept_cnt", "k_packed", "v_packed", "status", "workspace")):
        if t is not None:
            _out(t, numel, dtype, name)
    _check(_lib.compactor_compress(pp, arr, n, _ptr(scores), _ptr(kept_idx), _ptr(kept_cnt),
                                   _ptr(k_packed), _ptr(v_packed), _ptr(status), _ptr(workspace),
                                   workspace.numel(), _stream(stream)))
    return {"scores": scores, "kept_idx": kept_idx, "kept_cnt": kept_cnt, "k_packed": k_packed,
            "v_packed": v_packed, "status": status, "workspace": workspace}


STATIC_SCRATCH_BYTES = 64 << 20      # COMPACTOR_STATIC_SCRATCH_BYTES of the header


def compactor_compress_static(params: Params, reqs: Sequence[Request], scores, kept_idx, kept_cnt,
                              k_packed, v_packed, status, stream=None):
    """compactor_compress on the library's own static scratch: every buffer is the caller's (none
    is allocated here, `scores` may be None) and no workspace is passed."""
    pp, arr, n = call = _marshal(params, reqs, on_gpu=False)
    so, ko, _ = _layout(*call)
    nh = n * params.layers * params.kv_heads
    _check_gpu(params, reqs)
    _out(scores, so[-1], torch.float32, "scores")
    for t, name in ((kept_idx, "kept_idx"), (kept_cnt, "kept_cnt"), (k_packed, "k_packed"),
                    (v_packed, "v_packed"), (status, "status")):
        _require(t is not None, "%s must be supplied" % name)
    _out(kept_idx, ko[-1], torch.int32, "kept_idx")
    _out(kept_cnt, nh, torch.int32, "kept_cnt")
    _out(k_packed, ko[-1] * params.head_dim, torch.bfloat16, "k_packed")
    _out(v_packed, ko[-1] * params.head_dim, torch.bfloat16, "v_packed")
    _out(status, nh, torch.int32, "status")
    _check(_lib.compactor_compress_static(pp, arr, n, _ptr(scores), _ptr(kept_idx), _ptr(kept_cnt),
                                          _ptr(k_packed), _ptr(v_packed), _ptr(status),
                                          _stream(stream)))


@dataclass
class AttnParams:
    layers: int
    kv_heads: int
    q_heads: int
    head_dim: int = 128
    chunk: int = 256
    pool: int = 7
    scale: float = 0.0          # 0 = 1/sqrt(head_dim)

    def c(self) -> _AttnParams:
        return _AttnParams(self.layers, self.kv_heads, self.q_heads, self.head_dim, self.chunk,
                           self.pool, self.scale)


@dataclass
class AttnRequest:
    q: torch.Tensor             # bf16 [L, Hq, n, d]
    k: torch.Tensor             # bf16 [L, H, n, d]

    def c(self, params: Optional["AttnParams"] = None) -> _AttnRequest:
        q, k = self.q, self.k
        _require(q.dtype == torch.bfloat16 and k.dtype == torch.bfloat16, "q and k must be bfloat16")
        _require(q.dim() == 4 and k.dim() == 4 and q.stride(3) == 1 and k.stride(3) == 1,
                 "q and k must be [L, heads, n, d] with d contiguous")
        qs, ks = tuple(q.shape), tuple(k.shape)
        _require(qs[2] == ks[2], "q and k must cover the same tokens")
        if params is not None and not (qs[:2] == (params.layers, params.q_heads) and
                                       ks[:2] == (params.layers, params.kv_heads) and
                                       qs[3] == params.head_dim and ks[3] == params.head_dim):
            _refuse("q %s / k %s do not match the parameters [%d, %d | %d, n, %d]"
                    % (qs, ks, params.layers, params.q_heads, params.kv_heads, params.head_dim))
        _require(q.is_cuda and k.is_cuda, "q and k must live on the GPU")
        return _AttnRequest(q.data_ptr(), k.data_ptr(), *q.stride()[:3], *k.stride()[:3], ks[2])


def compactor_attention_workspace_size(params: AttnParams, reqs: Sequence[AttnRequest]) -> int:
    arr = (_AttnRequest * len(reqs))(*[r.c(params) for r in reqs])
    out = C.c_size_t(0)
    _check(_lib.compactor_attention_workspace_size(C.byref(params.c()), arr, len(reqs), C.byref(out)))
    return int(out.value)


def compactor_attention_scores(params: AttnParams, reqs: Sequence[AttnRequest], attn=None,
                               workspace=None, stream=None):
    """-> attn fp32 [sum_b L*H*n_b]; request b starts at the prefix sum of L*H*n_b."""
    dev = reqs[0].k.device
    total = sum(params.layers * params.kv_heads * r.k.shape[2] for r in reqs)
    given = attn, workspace                    # what is allocated here needs no check
    if attn is None:
        attn = _empty(stream, total, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _empty(stream, max(256, compactor_attention_workspace_size(params, reqs)), returned=False,
                           dtype=torch.uint8, device=dev)
    arr = (_AttnRequest * len(reqs))(*[r.c(params) for r in reqs])
    _out(given[0], total, torch.float32, "attn")
    _out(given[1], 0, torch.uint8, "workspace")
    _check(_lib.compactor_attention_scores(C.byref(params.c()), arr, len(reqs), _ptr(attn),
                                           _ptr(workspace), workspace.numel(), _stream(stream)))
    return attn


class Cache:
    """The caches of some contexts in one page pool, for the calls that serve from them (see
    compactor_cache_t).  Checked once, here; the tensors stay the caller's, and must not be resized
    or moved while the Cache is in use.

    k_pages, v_pages  bf16 views indexed [page, layer, slot, head, channel], as compactor_compact_paged
                      takes them
    tables            int32 [request, logical page]
    counts            int32 [request, layer, head]: tokens that each head holds
    seen              int32, same shape and strides: tokens it has ever been given
    mass, positions   fp32 and int32 views indexed [page, layer, head, slot], slots contiguous
    seen, mass and positions: all three, or none."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, tables: torch.Tensor,
                 counts: torch.Tensor, seen: Optional[torch.Tensor] = None,
                 mass: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None):
        self._c = self._take(k_pages, v_pages, torch.bfloat16, tables, counts, seen, mass, positions)
        self._c.head_dim = k_pages.shape[4]
        self._ref = self._plain = C.byref(self._c)

    def _take(self, k_pages, v_pages, dtype, tables, counts, seen, mass, positions) -> _Cache:
        if k_pages.dtype != dtype or v_pages.dtype != dtype:
            _refuse("k_pages and v_pages must be %s" % str(dtype).split(".")[1])
        _require(k_pages.dim() == 5 and k_pages.stride(4) == 1 and v_pages.shape == k_pages.shape and
                 v_pages.stride() == k_pages.stride(),
                 "k_pages and v_pages must be [page, layer, slot, head, channel] views of equal shape and "
                 "strides, channel contiguous")
        pages, layers, page_size, heads, _ = k_pages.shape
        _require(tables.dtype == torch.int32 and tables.dim() == 2 and tables.shape[0] >= 1 and
                 tables.shape[1] >= 1 and (tables.stride(1) == 1 or tables.shape[1] == 1),
                 "tables must be int32 [request, logical page], logical pages contiguous")
        nreq, table_len = tables.shape
        _require(nreq == 1 or tables.stride(0) >= table_len, "the tables of two requests must not overlap")
        _require((seen is None) == (mass is None) == (positions is None) and (seen is None or mass is not None),
                 "seen, mass and positions: all three, or none")
        for name, t in (("counts", counts), ("seen", seen)):
            if t is not None and not (t.dtype == torch.int32 and tuple(t.shape) == (nreq, layers, heads) and
                                      (t.stride(2) == 1 or heads == 1) and t.stride() == counts.stride()):
                _refuse("%s must be int32 [request, layer, head] = [%d, %d, %d], heads contiguous, with the "
                        "strides of counts" % (name, nreq, layers, heads))
        for name, t, dtype in (("mass", mass, torch.float32), ("positions", positions, torch.int32)):
            if t is not None and not (t.dtype == dtype and tuple(t.shape) == (pages, layers, heads, page_size) and
                                      (t.stride(3) == 1 or page_size == 1) and t.stride() == mass.stride()):
                _refuse("%s must be %s [page, layer, head, slot] = [%d, %d, %d, %d], slots contiguous, with the "
                        "strides of mass" % (name, dtype, pages, layers, heads, page_size))
        for name, t in (("k_pages", k_pages), ("counts", counts), ("seen", seen), ("mass", mass), ("positions", positions)):
            if t is not None and any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
                _refuse("%s is written: its elements must not share memory" % name)
        self.device = k_pages.device
        for name, t in (("k_pages", k_pages), ("v_pages", v_pages), ("tables", tables), ("counts", counts),
                        ("seen", seen), ("mass", mass), ("positions", positions)):
            if t is not None and not t.is_cuda:
                _refuse("%s must live on the GPU" % name)
            if t is not None and t.device != self.device:
                _refuse("%s must live on the GPU of the page pool" % name)
        self.k_pages, self.v_pages, self.tables, self.counts = k_pages, v_pages, tables, counts
        self.seen, self.mass, self.positions = seen, mass, positions
        self.nreq, self.layers, self.kv_heads = nreq, layers, heads
        self._bytes = {}              # workspace sizes
        pool = _PagePool(k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1),
                         k_pages.stride(3), k_pages.stride(2), page_size, pages)
        st = mass.stride() if mass is not None else (0, 0, 0)
        return _Cache(pool, tables.data_ptr(), max(tables.stride(0), table_len), table_len, nreq, layers, heads, 128,
                      counts.data_ptr(), _ptr(seen), counts.stride(0), counts.stride(1), _ptr(mass), _ptr(positions),
                      st[0], st[1], st[2])

    def layer(self, first: int, count: int = 1) -> "Cache":
        """The cache of `count` layers from `first` on, for calls layer by layer."""
        _require(0 <= first and count >= 1 and first + count <= self.layers, "no such layers")
        at = slice(first, first + count)
        some = lambda t: None if t is None else t[:, at]      # noqa: E731
        part = type(self)(self.k_pages[:, at], self.v_pages[:, at], *[some(t) for t in self._scales], self.tables, self.counts[:, at],
                          some(self.seen), some(self.mass), some(self.positions))
        part._whole = self._whole and count == self.layers
        return part

    _scales = ()
    _whole = True                 # of all the layers that share the tables

    def _new_tokens(self, t: Optional[torch.Tensor]) -> int:
        if t is None:
            return 0
        if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != self.nreq or not t.is_contiguous():
            _refuse("new_tokens must be a contiguous int32 tensor of %d requests" % self.nreq)
        if t.device != self.device:
            _refuse("new_tokens must live on the GPU of the cache")
        return t.data_ptr()

    def _workspace(self, size, what, key, given, stream):
        """-> (pointer, bytes), and the tensor that holds them.  key: what the size depends on beside the cache's own sizes."""
        if given is not None:
            _out(given, 0, torch.uint8, "workspace")
            if given.device != self.device:
                _refuse("the workspace must live on the GPU of the cache")
            return given.data_ptr(), given.numel(), given
        need = self._bytes.get(key)
        if need is None:
            out = C.c_size_t(0)
            _check(size(self._ref, what, C.byref(out)))
            need = self._bytes[key] = out.value
        if need == 0:
            return 0, 0, None
        given = _empty(stream, need, returned=False, dtype=torch.uint8, device=self.device)
        return given.data_ptr(), need, given

    def _on(self, stream, call):
        """call(stream handle) with the cache's GPU current."""
        if stream is not None and stream.device != self.device:
            _refuse("the stream belongs to another GPU than the cache")
        here = torch.cuda.current_device()
        if here == self.device.index:
            _check(call(_stream(stream) if stream is not None or _raw_stream is None else _raw_stream(here)))
        else:
            with torch.cuda.device(self.device):
                _check(call(_stream(stream)))


class MxCache(Cache):
    """A Cache in 4 bits (see compactor_mx_cache_t), for the compactor_mx_* calls and those that take either kind.

    k_pages, v_pages    uint8 views indexed [page, layer, slot, head, byte], 64 bytes a row, contiguous
    k_scales, v_scales  uint8 views indexed [page, layer, head, slot, group], 4 bytes a slot, slots contiguous, both with the same
                        strides: four times those of mass
    The others as in Cache."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor,
                 tables: torch.Tensor, counts: torch.Tensor, seen: Optional[torch.Tensor] = None,
                 mass: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None):
        cache = self._take(k_pages, v_pages, torch.uint8, tables, counts, seen, mass, positions)
        pages, layers, page_size, heads, width = k_pages.shape
        if width != 64:
            _refuse("a row of k_pages must have 64 bytes, got %d" % width)
        st = k_scales.stride()
        for name, t in (("k_scales", k_scales), ("v_scales", v_scales)):
            if (t.dtype != torch.uint8 or tuple(t.shape) != (pages, layers, heads, page_size, 4) or t.stride() != st or
                    st[4] != 1 or (st[3] != 4 and page_size > 1) or any(x % 4 for x in st[:3])):
                _refuse("%s must be uint8 [page, layer, head, slot, group] = [%d, %d, %d, %d, 4], slots of 4 bytes one behind the other, "
                        "with the strides of k_scales" % (name, pages, layers, heads, page_size))
            if any(n > 1 and x == 0 for n, x in zip(t.shape, st)):
                _refuse("%s is written: its elements must not share memory" % name)
            if t.device != self.device or not t.is_cuda:
                _refuse("%s must live on the GPU of the page pool" % name)
        if mass is not None and any(n > 1 and x != 4 * y for n, x, y in zip(mass.shape, st, mass.stride())):
            _refuse("the strides of k_scales must be four times those of mass")
        cache.state_page_stride, cache.state_layer_stride, cache.state_head_stride = (x // 4 for x in st[:3])
        self.k_scales, self.v_scales = self._scales = k_scales, v_scales
        self._mx = _MxCache(cache, k_scales.data_ptr(), v_scales.data_ptr())
        self._c = self._mx.cache
        self._ref, self._plain = C.byref(self._mx), C.byref(self._c)      # (_plain: for calls that look at no rows)


def _either(cache, mx: bool):
    """The calls of one kind of rows do not read the other."""
    if isinstance(cache, MxCache) != mx:
        _refuse("this call is for a cache of %s bits" % ("4" if mx else "16"))


def compactor_cache_admit(params: Params, reqs: Sequence[Request], kept_idx: torch.Tensor,
                          kept_cnt: torch.Tensor, cache: Cache, scores: Optional[torch.Tensor] = None,
                          stream=None):
    """State of the rows that compactor_compact_paged has written into the cache's pages: counts, seen,
    positions and, from the scores, mass."""
    _either(cache, False)
    n = len(reqs)
    _require(n >= 1, "at least one request is needed")
    arr = (_Request * n)()                     # n and ratio are all that is looked at
    layers, heads = params.layers, params.kv_heads
    for r, a in zip(reqs, arr):
        L, H, a.n, _d = r.k_score.shape
        if L != layers or H != heads:
            _refuse("k_score has shape %s, the parameters say [%d, %d, n, %d]"
                    % (tuple(r.k_score.shape), params.layers, params.kv_heads, params.head_dim))
        a.ratio = r.ratio
    pp = C.byref(params.c(False))
    so, ko, kk = (C.c_int64 * (n + 1))(), (C.c_int64 * (n + 1))(), (C.c_int32 * n)()
    _check(_lib.compactor_layout(pp, arr, n, so, ko, kk))
    if (n, params.layers, params.kv_heads) != (cache.nreq, cache.layers, cache.kv_heads):
        _refuse("the cache is of [%d, %d, %d] requests, layers and heads, the call of [%d, %d, %d]"
                % (cache.nreq, cache.layers, cache.kv_heads, n, params.layers, params.kv_heads))
    for t, numel, dtype, name in ((kept_idx, ko[n], torch.int32, "kept_idx"),
                                  (kept_cnt, n * params.layers * params.kv_heads, torch.int32, "kept_cnt"),
                                  (scores, so[n], torch.float32, "scores")):
        _out(t, numel, dtype, name)
        if t is not None and t.device != cache.device:
            _refuse("%s must live on the GPU of the cache" % name)
    cache._on(stream, lambda st: _lib.compactor_cache_admit(pp, arr, n, _ptr(kept_idx), _ptr(kept_cnt), _ptr(scores),
                                                            cache._ref, st))


def compactor_cache_append(cache: Cache, k: torch.Tensor, v: torch.Tensor,
                           new_tokens: Optional[torch.Tensor] = None, stream=None):
    """Rows of new tokens into the cache.  k, v: bf16 [request, layer, token, kv head, channel], any
    strides with the channel contiguous, the same for both; new_tokens: int32 [request], how many of
    its rows each request brings (None: all)."""
    _either(cache, False)
    rows = _rows(cache, k, v, new_tokens)
    cache._on(stream, lambda st: _lib.compactor_cache_append(cache._ref, C.byref(rows), st))


def _rows(cache: Cache, k, v, new_tokens) -> _CacheRows:
    if k.dtype != torch.bfloat16 or k.dim() != 5 or v.dtype != torch.bfloat16:
        _refuse("k and v must be bfloat16 [request, layer, token, head, channel]")
    B, L, T, H, d = k.shape
    sb, sl, st_, sh, sc = k.stride()
    if (B, L, H, d) != (cache.nreq, cache.layers, cache.kv_heads, cache._c.head_dim):
        _refuse("k has shape %s, the cache is of [%d, %d, tokens, %d, %d]"
                % (tuple(k.shape), cache.nreq, cache.layers, cache.kv_heads, cache._c.head_dim))
    if sc != 1 or v.shape != k.shape or v.stride() != (sb, sl, st_, sh, sc):
        _refuse("v must have the shape and strides of k, the channel contiguous")
    if k.device != cache.device or v.device != cache.device:
        _refuse("k and v must live on the GPU of the cache")
    _int32(tokens=T)
    return _CacheRows(k.data_ptr(), v.data_ptr(), sb, sl, st_, sh, cache._new_tokens(new_tokens), T)


def _cache_query(cache: Cache, q, new_tokens, scale, softcap, accumulate, max_tokens):
    if q.dtype != torch.bfloat16 or q.dim() != 5:
        _refuse("q must be bfloat16 [request, layer, token, query head, channel]")
    B, L, T, Hq, d = q.shape
    sb, sl, st, sh, sc = q.stride()
    if (B, L, d) != (cache.nreq, cache.layers, cache._c.head_dim) or sc != 1:
        _refuse("q has shape %s and strides %s, the cache is of [%d, %d, tokens, query heads, %d], the channel contiguous"
                % (tuple(q.shape), q.stride(), cache.nreq, cache.layers, cache._c.head_dim))
    if q.device != cache.device:
        _refuse("q must live on the GPU of the cache")
    _int32(max_tokens=max_tokens)
    return _CacheQuery(q.data_ptr(), 0, 0, sb, sl, st, sh, 0, 0, 0, 0, cache._new_tokens(new_tokens), T, Hq, scale,
                       softcap, 1 if accumulate else 0, max_tokens)


def _attention_bytes(call, cache, q, accumulate, max_tokens) -> int:
    out = C.c_size_t(0)
    query = _cache_query(cache, q, None, 0.0, 0.0, accumulate, max_tokens)
    _check(call(cache._ref, C.byref(query), C.byref(out)))
    return int(out.value)


def compactor_cache_attention_workspace_size(cache: Cache, q: torch.Tensor, accumulate: bool = False,
                                             max_tokens: int = 0) -> int:
    _either(cache, False)
    return _attention_bytes(_lib.compactor_cache_attention_workspace_size, cache, q, accumulate, max_tokens)


def compactor_cache_attention(cache: Cache, q: torch.Tensor, new_tokens: Optional[torch.Tensor] = None,
                              scale: float = 0.0, softcap: float = 0.0, accumulate: bool = False,
                              max_tokens: int = 0, want_lse: bool = False, out=None, lse=None,
                              workspace=None, stream=None):
    """Attention of the tokens appended last to the cache.  q: bf16 [request, layer, token, query head,
    channel], any strides with the channel contiguous; out must not be the memory of q.  -> (out, bf16 of q's shape; lse, fp32
    [request, layer, token, query head], or None unless asked for or given)"""
    _either(cache, False)
    return _attention(_lib.compactor_cache_attention, _lib.compactor_cache_attention_workspace_size, cache, q, new_tokens, scale,
                      softcap, accumulate, max_tokens, want_lse, out, lse, workspace, stream)


def _attention(call, size, cache, q, new_tokens, scale, softcap, accumulate, max_tokens, want_lse, out, lse, workspace, stream):
    query = _cache_query(cache, q, new_tokens, scale, softcap, accumulate, max_tokens)
    shape = q.shape
    if out is None:
        out = _made_on(stream, lambda: torch.empty_like(q))      # (half of what torch.empty with a device takes)
        if out.stride(4) != 1:
            out = _empty(stream, shape, dtype=torch.bfloat16, device=cache.device)
    else:
        if out.dtype != torch.bfloat16 or out.shape != shape or out.stride(4) != 1 or out.device != cache.device:
            _refuse("out must be bfloat16 of q's shape on the GPU of the cache, the channel contiguous")
        if any(n > 1 and s == 0 for n, s in zip(shape, out.stride())):
            _refuse("out is written: its elements must not share memory")
    query.out = out.data_ptr()
    query.out_stride_b, query.out_stride_l, query.out_stride_t, query.out_stride_h, _ = out.stride()
    if lse is not None:
        _out(lse, shape[0] * shape[1] * shape[2] * shape[3], torch.float32, "lse")
        if lse.device != cache.device:
            _refuse("lse must live on the GPU of the cache")
    elif want_lse:
        lse = _made_on(stream, lambda: q.new_empty(shape[:4], dtype=torch.float32))
    query.lse = _ptr(lse)
    ref = C.byref(query)
    ptr, nbytes, _keep = cache._workspace(size, ref, (shape[2], shape[3], accumulate, max_tokens), workspace, stream)
    cache._on(stream, lambda st: call(cache._ref, ref, ptr, nbytes, st))
    return out, lse


def _cache_evict(cache: Cache, budget, budgets, sink, recent, scope, max_tokens):
    if (budget is None) == (budgets is None):
        _refuse("either budget or budgets")
    ptr = 0
    if budgets is not None:
        if budgets.dtype != torch.int32 or tuple(budgets.shape) != (cache.nreq,) or not budgets.is_contiguous():
            _refuse("budgets must be a contiguous int32 tensor of %d requests" % cache.nreq)
        if budgets.device != cache.device:
            _refuse("budgets must live on the GPU of the cache")
        ptr = budgets.data_ptr()
    budget = 0 if budget is None else budget
    _int32(budget=budget, sink=sink, recent=recent, max_tokens=max_tokens)
    return _CacheEvict(budget, ptr, sink, recent, scope, max_tokens)


def _evict_bytes(call, cache, scope, max_tokens) -> int:
    out = C.c_size_t(0)
    _int32(max_tokens=max_tokens)
    evict = _CacheEvict(0, 0, 0, 0, scope, max_tokens)
    _check(call(cache._ref, C.byref(evict), C.byref(out)))
    return int(out.value)


def compactor_cache_evict_workspace_size(cache: Cache, scope: int = SCOPE_HEAD, max_tokens: int = 0) -> int:
    _either(cache, False)
    return _evict_bytes(_lib.compactor_cache_evict_workspace_size, cache, scope, max_tokens)


def compactor_cache_evict(cache: Cache, budget: Optional[int] = None, budgets: Optional[torch.Tensor] = None,
                          sink: int = 0, recent: int = 0, scope: int = SCOPE_HEAD, max_tokens: int = 0,
                          workspace=None, stream=None):
    """Brings every head (SCOPE_LAYER: the heads of every layer together) down to its budget: `budget`
    tokens, or budgets[request] of an int32 device tensor."""
    _either(cache, False)
    _evict(_lib.compactor_cache_evict, _lib.compactor_cache_evict_workspace_size, cache, budget, budgets, sink, recent, scope,
           max_tokens, workspace, stream)


def _evict(call, size, cache, budget, budgets, sink, recent, scope, max_tokens, workspace, stream):
    ref = C.byref(_cache_evict(cache, budget, budgets, sink, recent, scope, max_tokens))
    ptr, nbytes, _keep = cache._workspace(size, ref, (scope, max_tokens), workspace, stream)
    cache._on(stream, lambda st: call(cache._ref, ref, ptr, nbytes, st))


def compactor_mx_append(cache: MxCache, k: torch.Tensor, v: torch.Tensor,
                         new_tokens: Optional[torch.Tensor] = None, stream=None):
    """compactor_cache_append into a cache in 4 bits: k and v are bfloat16, as there."""
    _either(cache, True)
    rows = _rows(cache, k, v, new_tokens)
    cache._on(stream, lambda st: _lib.compactor_mx_append(cache._ref, C.byref(rows), st))


def compactor_mx_store(cache: MxCache, source: Cache, stream=None):
    """Makes of `cache` what `source`, a cache of 16 bits of as many requests, layers and heads, holds."""
    _either(cache, True)
    _either(source, False)
    if (source.nreq, source.layers, source.kv_heads) != (cache.nreq, cache.layers, cache.kv_heads):
        _refuse("the source is of [%d, %d, %d] requests, layers and heads, the cache of [%d, %d, %d]"
                % (source.nreq, source.layers, source.kv_heads, cache.nreq, cache.layers, cache.kv_heads))
    _require(cache.mass is None or source.mass is not None, "a cache with state needs a source with state")
    _require(source.device == cache.device, "the source must live on the GPU of the cache")
    cache._on(stream, lambda st: _lib.compactor_mx_store(cache._ref, source._ref, st))


def compactor_mx_read(cache: MxCache, tokens: int, first: Optional[int] = None, new_tokens: Optional[torch.Tensor] = None,
                       k=None, v=None, stream=None):
    """Rows of `tokens` slots from `first` on (None: those that were appended last, with new_tokens those of each request) as
    bfloat16, zeros where there are none.  -> (k, v) [request, layer, token, kv head, channel]; given ones may have any
    strides with the channel contiguous, the same for both."""
    _either(cache, True)
    _int32(tokens=tokens)
    shape = (cache.nreq, cache.layers, tokens, cache.kv_heads, 128)
    if (k is None) != (v is None):
        _refuse("k and v: both, or none")
    if k is None:
        make = lambda: cache.counts.new_empty(shape, dtype=torch.bfloat16)      # noqa: E731 (half of what torch.empty with a device takes)
        k, v = _made_on(stream, make), _made_on(stream, make)
    else:
        for t in (k, v):
            if t.dtype != torch.bfloat16 or tuple(t.shape) != shape or t.stride() != k.stride() or t.stride(4) != 1:
                _refuse("k and v must be bfloat16 %s with the same strides, the channel contiguous" % (shape,))
            if t.device != cache.device:
                _refuse("k and v must live on the GPU of the cache")
            if any(n > 1 and s == 0 for n, s in zip(shape, t.stride())):
                _refuse("k and v are written: their elements must not share memory")
    if first is not None:
        _int32(first=first)
    rows = _CacheRowsOut(k.data_ptr(), v.data_ptr(), *k.stride()[:4], cache._new_tokens(new_tokens), tokens, -1 if first is None else first)
    cache._on(stream, lambda st: _lib.compactor_mx_read(cache._ref, C.byref(rows), st))
    return k, v


def compactor_mx_attention_workspace_size(cache: MxCache, q: torch.Tensor, accumulate: bool = False, max_tokens: int = 0) -> int:
    _either(cache, True)
    return _attention_bytes(_lib.compactor_mx_attention_workspace_size, cache, q, accumulate, max_tokens)


def compactor_mx_attention(cache: MxCache, q: torch.Tensor, new_tokens: Optional[torch.Tensor] = None,
                            scale: float = 0.0, softcap: float = 0.0, accumulate: bool = False,
                            max_tokens: int = 0, want_lse: bool = False, out=None, lse=None,
                            workspace=None, stream=None):
    """compactor_cache_attention, to a cache in 4 bits."""
    _either(cache, True)
    return _attention(_lib.compactor_mx_attention, _lib.compactor_mx_attention_workspace_size, cache, q, new_tokens, scale,
                      softcap, accumulate, max_tokens, want_lse, out, lse, workspace, stream)


def compactor_mx_evict_workspace_size(cache: MxCache, scope: int = SCOPE_HEAD, max_tokens: int = 0) -> int:
    _either(cache, True)
    return _evict_bytes(_lib.compactor_mx_evict_workspace_size, cache, scope, max_tokens)


def compactor_mx_evict(cache: MxCache, budget: Optional[int] = None, budgets: Optional[torch.Tensor] = None,
                        sink: int = 0, recent: int = 0, scope: int = SCOPE_HEAD, max_tokens: int = 0,
                        workspace=None, stream=None):
    """compactor_cache_evict, from a cache in 4 bits."""
    _either(cache, True)
    _evict(_lib.compactor_mx_evict, _lib.compactor_mx_evict_workspace_size, cache, budget, budgets, sink, recent, scope,
           max_tokens, workspace, stream)


class Rotation:
    """Norms and rotary positions of the heads of some layers (see compactor_rotation_t).  Checked once, here; the tensors stay the caller's.

    freqs           float64 [rotary_dim / 2]: radians per position of each pair of channels
    rotary_dim      channels that are rotated (None: twice as many as freqs); interleaved: pairs of neighbours, else of halves
    q_norm, k_norm  float32 [layer, 128]: weights of the norms, None where there is none; eps: theirs"""

    def __init__(self, freqs: torch.Tensor, rotary_dim: Optional[int] = None, interleaved: bool = False,
                 q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6):
        rotary_dim = 2 * freqs.numel() if rotary_dim is None else rotary_dim
        if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous() or 2 * freqs.numel() != rotary_dim:
            _refuse("freqs must be a contiguous float64 tensor of rotary_dim / 2 = %s / 2 numbers" % rotary_dim)
        if not 8 <= rotary_dim <= 128 or rotary_dim % 8:
            _refuse("rotary_dim must be a multiple of 8 from 8 to 128, got %s" % rotary_dim)
        self.device, self.layers = freqs.device, None
        for name, t in (("q_norm", q_norm), ("k_norm", k_norm)):
            if t is None:
                continue
            if t.dtype != torch.float32 or t.dim() != 2 or t.shape[1] != 128 or not t.is_contiguous():
                _refuse("%s must be a contiguous float32 tensor [layers, 128]" % name)
            if self.layers not in (None, t.shape[0]):
                _refuse("q_norm and k_norm must be of as many layers")
            if t.device != self.device:
                _refuse("%s must live on the GPU of freqs" % name)
            self.layers = t.shape[0]
        _require(freqs.is_cuda, "freqs must live on the GPU")
        self.freqs, self.rotary_dim, self.interleaved = freqs, rotary_dim, interleaved
        self.q_norm, self.k_norm, self.eps = q_norm, k_norm, eps
        self._c = _Rotation(freqs.data_ptr(), rotary_dim, 1 if interleaved else 0, _ptr(q_norm), _ptr(k_norm), eps)
        self._ref = C.byref(self._c)

    def layer(self, first: int, count: int = 1) -> "Rotation":
        """That of `count` layers from `first` on, for calls layer by layer."""
        _require(self.layers is None or (0 <= first and count >= 1 and first + count <= self.layers), "no such layers")
        some = lambda t: None if t is None else t[first:first + count]      # noqa: E731
        return Rotation(self.freqs, self.rotary_dim, self.interleaved, some(self.q_norm), some(self.k_norm), self.eps)

    def _fits(self, layers: int, device):
        if self.layers not in (None, layers):
            _refuse("the norms are of %s layers, the rows of %s" % (self.layers, layers))
        if self.device != device:
            _refuse("the rotation and the rows must live on the same GPU")


def _head_rows(t, what, shape=None, device=None):
    if t.dtype != torch.bfloat16 or t.dim() != 5 or t.stride(4) != 1 or t.shape[4] != 128:
        _refuse("%s must be bfloat16 [request, layer, token, head, 128], the channel contiguous" % what)
    if shape is not None and t.shape != shape:
        _refuse("%s has shape %s, %s is needed" % (what, tuple(t.shape), tuple(shape)))
    if device is not None and t.device != device:
        _refuse("%s must live on the GPU of the others" % what)


def _head_rows_out(t, like, what, stream):
    """A given output, or a new one."""
    if t is None:
        t = _made_on(stream, lambda: torch.empty_like(like))
        return t if t.stride(4) == 1 else _empty(stream, like.shape, dtype=torch.bfloat16, device=like.device)
    _head_rows(t, what, like.shape, like.device)
    if any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
        _refuse("%s is written: its elements must not share memory" % what)
    return t


def _on_gpu(device, stream, call):
    """call(stream handle) with the tensors' GPU current."""
    if stream is not None and stream.device != device:
        _refuse("the stream belongs to another GPU than the rows")
    if device.index in (None, torch.cuda.current_device()):
        _check(call(_stream(stream)))
    else:
        with torch.cuda.device(device):
            _check(call(_stream(stream)))


def compactor_rotate(rotation: Rotation, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor,
                     new_tokens: Optional[torch.Tensor] = None, want_plain: bool = False, q_out=None, k_out=None, k_plain=None,
                     stream=None):
    """Queries and keys normed and rotated by position.  q, k: bf16 [request, layer, token, head, 128], any strides with the channel
    contiguous, one of them may be None; positions: int32 [request, token], or [token] for all requests; q_out, k_out: other
    memory, or q and k themselves.  -> (q, k, keys before the rotation, or None unless asked for or given)"""
    rows = q if q is not None else k
    _require(rows is not None, "q or k is needed")
    for name, t in (("q", q), ("k", k)):
        if t is not None:
            _head_rows(t, name, None, rows.device)
            _require(t.is_cuda, "q and k must live on the GPU")
            if t.shape[:3] != rows.shape[:3]:
                _refuse("q and k must be of the same requests, layers and tokens")
    B, L, T = rows.shape[:3]
    rotation._fits(L, rows.device)
    if positions.dtype != torch.int32 or tuple(positions.shape) not in ((B, T), (T,)) or (positions.stride(-1) != 1 and T > 1):
        _refuse("positions must be int32 [%d, %d] or [%d], tokens contiguous" % (B, T, T))
    if new_tokens is not None and (new_tokens.dtype != torch.int32 or tuple(new_tokens.shape) != (B,) or not new_tokens.is_contiguous()):
        _refuse("new_tokens must be a contiguous int32 tensor of %d requests" % B)
    for name, t in (("positions", positions), ("new_tokens", new_tokens)):
        if t is not None and t.device != rows.device:
            _refuse("%s must live on the GPU of the rows" % name)
    if k is None and (want_plain or k_plain is not None or k_out is not None) or q is None and q_out is not None:
        _refuse("an output without its rows")
    if q is not None:
        q_out = _head_rows_out(q_out, q, "q_out", stream)
    if k is not None:
        k_out = _head_rows_out(k_out, k, "k_out", stream)
        if want_plain or k_plain is not None:
            k_plain = _head_rows_out(k_plain, k, "k_plain", stream)
    tensors = q, k, q_out, k_out, k_plain
    strides = [s for t in tensors for s in (t.stride()[:4] if t is not None else (0, 0, 0, 0))]
    c = _RotateRows(*[_ptr(t) for t in tensors], *strides, positions.data_ptr(), positions.stride(0) if positions.dim() == 2 and B > 1 else 0,
                    _ptr(new_tokens), B, L, T, q.shape[3] if q is not None else 0, k.shape[3] if k is not None else 0)
    _on_gpu(rows.device, stream, lambda st: _lib.compactor_rotate(rotation._ref, C.byref(c), st))
    return q_out, k_out, k_plain


def compactor_cache_append_rotated(cache: Cache, rotation: Rotation, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
                                   new_tokens: Optional[torch.Tensor] = None, q_out=None, stream=None):
    """compactor_cache_append of keys that are normed and rotated on the way, to the positions that they get, and the queries of the
    same tokens likewise.  -> q rotated (None without q); rows of padding tokens are left as they are, in new memory they hold anything"""
    _either(cache, False)
    return _append_rotated(_lib.compactor_cache_append_rotated, cache, rotation, k, v, q, new_tokens, q_out, stream)


def compactor_mx_append_rotated(cache: MxCache, rotation: Rotation, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
                                new_tokens: Optional[torch.Tensor] = None, q_out=None, stream=None):
    """compactor_cache_append_rotated, into a cache in 4 bits."""
    _either(cache, True)
    return _append_rotated(_lib.compactor_mx_append_rotated, cache, rotation, k, v, q, new_tokens, q_out, stream)


def _append_rotated(call, cache, rotation, k, v, q, new_tokens, q_out, stream):
    rows = _rows(cache, k, v, new_tokens)
    rotation._fits(cache.layers, cache.device)
    queries = None
    if q is not None:
        _head_rows(q, "q", None, cache.device)
        if q.shape[:3] != k.shape[:3]:
            _refuse("q and k must be of the same requests, layers and tokens")
        q_out = _head_rows_out(q_out, q, "q_out", stream)
        queries = C.byref(_RotateQueries(q.data_ptr(), q_out.data_ptr(), *q.stride()[:4], *q_out.stride()[:4], q.shape[3]))
    elif q_out is not None:
        _refuse("an output without its rows")
    cache._on(stream, lambda st: call(cache._ref, rotation._ref, C.byref(rows), queries, st))
    return q_out


def _pages(cache: Cache, *tensors):
    """Checks of the calls that change tables -> the cache, as they take it.  tensors: (name, tensor, shape), int32 and contiguous, or None"""
    if not cache._whole:
        _refuse("the pages are those of all layers: this call takes the cache that layer() was called on")
    device = cache.device
    for name, t, shape in tensors:
        if t is None:
            continue
        if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
            _refuse("%s must be a contiguous int32 tensor %s" % (name, list(shape)))
        if t.device != device:
            _refuse("%s must live on the GPU of the cache" % name)
    return cache._plain


def _pages_bytes(call, cache: Cache) -> int:
    need = cache._bytes.get(call.__name__)
    if need is None:
        out = C.c_size_t(0)
        _check(call(cache._plain, C.byref(out)))
        need = cache._bytes[call.__name__] = int(out.value)
    return need


def _pages_workspace(call, cache, given, stream):
    if given is None:
        need = _pages_bytes(call, cache)
        return _made_on(stream, lambda: cache.tables.new_empty(need, dtype=torch.uint8), False)      # (half of what torch.empty with a device takes)
    _out(given, 0, torch.uint8, "workspace")
    if given.device != cache.device:
        _refuse("the workspace must live on the GPU of the cache")
    return given


def _pages_out(cache, pairs, most, done, stream):
    if pairs is None:
        pairs = _made_on(stream, lambda: cache.tables.new_empty((most, 2)))
    if done is None:
        done = _made_on(stream, lambda: cache.tables.new_empty(2))
    return pairs, done


def compactor_pages_reserve_workspace_size(cache: Cache) -> int:
    return _pages_bytes(_lib.compactor_pages_reserve_workspace_size, cache)


def compactor_pages_compact_workspace_size(cache: Cache) -> int:
    return _pages_bytes(_lib.compactor_pages_compact_workspace_size, cache)


def compactor_pages_reserve(cache: Cache, refs: torch.Tensor, tokens: int, new_tokens: Optional[torch.Tensor] = None, own_all: bool = False,
                            pairs=None, done=None, workspace=None, stream=None):
    """Room for new tokens: entries of the tables that they need get free pages, pages that others name too are exchanged.  refs:
    int32 [page], how many times each is named, 0 a free one.  -> (pairs int32 [most, 2], done int32 [2]: how many pairs, how many pages were
    too few), for compactor_pages_copy.  cache: of 16 or 4 bits, here and in the calls below."""
    N = cache._c.pool.num_pages
    most = min(cache.nreq * cache._c.table_len, N)
    _int32(tokens=tokens)
    ref = _pages(cache, ("refs", refs, (N,)), ("pairs", pairs, (most, 2)), ("done", done, (2,)))
    pairs, done = _pages_out(cache, pairs, most, done, stream)
    ws = _pages_workspace(_lib.compactor_pages_reserve_workspace_size, cache, workspace, stream)
    c = _PagesReserve(refs.data_ptr(), cache._new_tokens(new_tokens), tokens, 1 if own_all else 0, pairs.data_ptr(), done.data_ptr())
    cache._on(stream, lambda st: _lib.compactor_pages_reserve(ref, C.byref(c), ws.data_ptr(), ws.numel(), st))
    return pairs, done


def _copy(call, cache, pairs, done, stream):
    _pages(cache, ("done", done, (2,)))
    if pairs.dtype != torch.int32 or pairs.dim() != 2 or pairs.shape[1] != 2 or pairs.shape[0] < 1 or not pairs.is_contiguous():
        _refuse("pairs must be a contiguous int32 tensor [most, 2]")
    if pairs.device != cache.device:
        _refuse("pairs must live on the GPU of the cache")
    cache._on(stream, lambda st: call(cache._ref, pairs.data_ptr(), pairs.shape[0], done.data_ptr(), st))


def compactor_pages_copy(cache: Cache, pairs: torch.Tensor, done: torch.Tensor, stream=None):
    """Copies the pages of the first done[0] pairs (from, to): rows of all layers and heads and their state."""
    _either(cache, False)
    _copy(_lib.compactor_pages_copy, cache, pairs, done, stream)


def compactor_mx_pages_copy(cache: MxCache, pairs: torch.Tensor, done: torch.Tensor, stream=None):
    """compactor_pages_copy, of a cache in 4 bits."""
    _either(cache, True)
    _copy(_lib.compactor_mx_pages_copy, cache, pairs, done, stream)


def compactor_pages_fork(cache: Cache, refs: torch.Tensor, parents: torch.Tensor, stream=None):
    """Request b goes on as request parents[b] was, on its pages.  parents: int32 [request]"""
    ref = _pages(cache, ("refs", refs, (cache._c.pool.num_pages,)), ("parents", parents, (cache.nreq,)))
    cache._on(stream, lambda st: _lib.compactor_pages_fork(ref, refs.data_ptr(), parents.data_ptr(), st))


def compactor_pages_release(cache: Cache, refs: torch.Tensor, finished: Optional[torch.Tensor] = None, stream=None):
    """Gives back the pages behind the last token of every request, and all of those that are finished (int32 [request], not 0)."""
    ref = _pages(cache, ("refs", refs, (cache._c.pool.num_pages,)), ("finished", finished, (cache.nreq,)))
    cache._on(stream, lambda st: _lib.compactor_pages_release(ref, refs.data_ptr(), _ptr(finished), st))


def compactor_pages_compact(cache: Cache, refs: torch.Tensor, pairs=None, done=None, workspace=None, stream=None):
    """Pushes the pages that are not free together to the lowest numbers.  -> (pairs int32 [most, 2], done int32 [2]: how many pairs, how many pages
    are not free), for compactor_pages_copy"""
    N = cache._c.pool.num_pages
    most = N // 2 + 1
    ref = _pages(cache, ("refs", refs, (N,)), ("pairs", pairs, (most, 2)), ("done", done, (2,)))
    pairs, done = _pages_out(cache, pairs, most, done, stream)
    ws = _pages_workspace(_lib.compactor_pages_compact_workspace_size, cache, workspace, stream)
    cache._on(stream, lambda st: _lib.compactor_pages_compact(ref, refs.data_ptr(), pairs.data_ptr(), done.data_ptr(), ws.data_ptr(), ws.numel(), st))
    return pairs, done


# The cache in 4 bits by the name of its numbers too: E2M1 codes are commonly called fp4, rows of them with E8M0 scales mx.
Fp4Cache = MxCache
compactor_fp4_append = compactor_mx_append
compactor_fp4_store = compactor_mx_store
compactor_fp4_read = compactor_mx_read
compactor_fp4_attention = compactor_mx_attention
compactor_fp4_attention_workspace_size = compactor_mx_attention_workspace_size
compactor_fp4_evict = compactor_mx_evict
compactor_fp4_evict_workspace_size = compactor_mx_evict_workspace_size
compactor_fp4_append_rotated = compactor_mx_append_rotated
compactor_fp4_pages_copy = compactor_mx_pages_copy
