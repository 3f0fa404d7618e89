"""Python binding of libtilemix.so (TileMix routed prefill attention for MI355X / gfx950).

Argument marshalling only: every step of the attention path runs in the HIP kernels of
libtilemix.so.  PyTorch provides device memory and streams.  The functions carry the names
of the C entry points declared in include/tilemix.h.  Importing this module does not load
the library; the first call does, and raises if it has not been built
(``python paper_2608_17336_amd/build.py`` or ``__graft_entry__.build()``).
"""

from __future__ import annotations

import ctypes
import math
import os
import struct
from dataclasses import dataclass
from typing import NamedTuple

__all__ = [
    "TilemixError",
    "Params",
    "library_path",
    "load_library",
    "tilemix_route_words_per_row",
    "tilemix_workspace_size",
    "tilemix_prefill",
    "tilemix_fused_workspace_size",
    "tilemix_prefill_fused",
    "tilemix_prefill_noalloc",
    "tilemix_prepare",
    "tilemix_attend",
    "tilemix_quantize",
    "tilemix_debug_qk_int32",
    "Template",
    "TEMPLATE_KINDS",
    "tilemix_auto_group_size",
    "tilemix_route_template",
    "tilemix_route_template_varlen",
    "tilemix_route_coverage",
    "tilemix_fit_template",
    "tilemix_varlen_workspace_size",
    "tilemix_prefill_varlen",
    "tilemix_varlen_fused_workspace_size",
    "tilemix_prefill_varlen_fused",
    "tilemix_debug_prefill",
    "tilemix_quantize_kv",
    "tilemix_decode_workspace_size",
    "tilemix_decode",
    "tilemix_decode_varlen",
    "PagedCache",
    "tilemix_paged_append",
    "tilemix_paged_gather",
    "tilemix_paged_decode_workspace_size",
    "tilemix_paged_decode",
    "PageList",
    "Reserved",
    "tilemix_paged_reserve",
    "tilemix_rotary_frequencies",
    "tilemix_rotary",
    "EXPORTED_SYMBOLS",
]

EXPORTED_SYMBOLS = (
    "tilemix_route_words_per_row",
    "tilemix_workspace_size",
    "tilemix_prefill",
    "tilemix_fused_workspace_size",
    "tilemix_prefill_fused",
    "tilemix_prefill_noalloc",
    "tilemix_prepare",
    "tilemix_attend",
    "tilemix_quantize",
    "tilemix_debug_qk_int32",
    "tilemix_auto_group_size",
    "tilemix_route_template",
    "tilemix_route_template_varlen",
    "tilemix_route_coverage",
    "tilemix_fit_template",
    "tilemix_varlen_workspace_size",
    "tilemix_prefill_varlen",
    "tilemix_varlen_fused_workspace_size",
    "tilemix_prefill_varlen_fused",
    "tilemix_debug_prefill",
    "tilemix_quantize_kv",
    "tilemix_decode_workspace_size",
    "tilemix_decode",
    "tilemix_decode_varlen",
    "tilemix_paged_append",
    "tilemix_paged_gather",
    "tilemix_paged_decode_workspace_size",
    "tilemix_paged_decode",
    "tilemix_paged_reserve",
    "tilemix_rotary_frequencies",
    "tilemix_rotary",
    "tilemix_status_string",
    "tilemix_last_error",
)

_HERE = os.path.dirname(os.path.abspath(__file__))


def library_path() -> str:
    return os.path.join(_HERE, "libtilemix.so")


class TilemixError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"tilemix status {status}: {message}")
        self.status = status


class _CParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("heads_q", ctypes.c_int32),
        ("heads_kv", ctypes.c_int32),
        ("len_q", ctypes.c_int32),
        ("len_k", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_m", ctypes.c_int32),
        ("block_n", ctypes.c_int32),
        ("group_size", ctypes.c_int32),
        ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("route_per_batch", ctypes.c_int32),
        ("route_hint", ctypes.c_int32),
    ]


@dataclass(frozen=True)
class Params:
    """Mirror of ``tilemix_params``."""
    batch: int
    heads_q: int
    heads_kv: int
    len_q: int
    len_k: int
    head_dim: int
    block_m: int = 128
    block_n: int = 64
    group_size: int = 1
    causal: bool = True
    scale: float = 0.0          # 0 -> 1/sqrt(head_dim)
    route_per_batch: bool = False
    route_hint: int = -1

    def c(self) -> _CParams:
        scale = self.scale if self.scale else 1.0 / math.sqrt(self.head_dim)
        return _CParams(self.batch, self.heads_q, self.heads_kv, self.len_q, self.len_k,
                        self.head_dim, self.block_m, self.block_n, self.group_size,
                        int(bool(self.causal)), scale, int(bool(self.route_per_batch)),
                        self.route_hint)

    @property
    def T_m(self) -> int:
        return -(-self.len_q // self.block_m)

    @property
    def T_n(self) -> int:
        return -(-self.len_k // self.block_n)


def _cparams(batch, heads_q, heads_kv, len_q, len_k, head_dim, tile, group_size, causal, scale,
             route_per_batch, route_hint) -> _CParams:
    """Params(...).c() without the dataclass in between (the calls' own path)."""
    return _CParams(batch, heads_q, heads_kv, len_q, len_k, head_dim, tile[0], tile[1], group_size,
                    1 if causal else 0, scale if scale else 1.0 / math.sqrt(head_dim),
                    1 if route_per_batch else 0, route_hint)


TEMPLATE_KINDS = {"one": 0, "zero": 1, "band": 2, "global": 3, "rowrand": 4, "aligned": 5,
                  "bigbird": 6, "sptrans": 7}


class _CTemplate(ctypes.Structure):
    _fields_ = [
        ("kind", ctypes.c_int32),
        ("band_w", ctypes.c_int32),
        ("global_groups", ctypes.c_int32),
        ("rand_fp16", ctypes.c_float),
        ("align_alpha", ctypes.c_float),
        ("align_beta", ctypes.c_float),
        ("sp_stride", ctypes.c_int32),
        ("sp_tail", ctypes.c_int32),
        ("seed", ctypes.c_uint64),
    ]


@dataclass(frozen=True)
class Template:
    """Mirror of ``tilemix_template`` (routing layouts of Appendix B)."""
    kind: str
    band_w: int = 0
    global_groups: int = 0
    rand_fp16: float = 0.0
    align_alpha: float = 0.0
    align_beta: float = 0.0
    sp_stride: int = 0
    sp_tail: int = 0
    seed: int = 0

    def c(self) -> _CTemplate:
        return _CTemplate(TEMPLATE_KINDS[self.kind], self.band_w, self.global_groups, self.rand_fp16,
                          self.align_alpha, self.align_beta, self.sp_stride, self.sp_tail, self.seed)

    @staticmethod
    def from_c(kind: str, t: _CTemplate) -> "Template":
        return Template(kind, t.band_w, t.global_groups, t.rand_fp16, t.align_alpha, t.align_beta,
                        t.sp_stride, t.sp_tail, t.seed)


class _CDebugExport(ctypes.Structure):
    _fields_ = [("q8", ctypes.c_void_p), ("dq", ctypes.c_void_p), ("tiles", ctypes.c_void_p),
                ("kinds", ctypes.c_void_p)]


_LIB = None


def load_library() -> ctypes.CDLL:
    """Load libtilemix.so (raises if it is missing: there is no fallback path).

    torch is imported first: its wheel carries its own HIP runtime under the same soname, and
    the library then binds to that one.  Loaded the other way round, the process would hold two
    HIP runtimes, and the library's would not see the device that torch's owns."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run __graft_entry__.build() first")
    try:
        import torch  # noqa: F401
    except ImportError:  # pragma: no cover - host-only use of the routing templates
        pass
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(_CParams)
    vp = ctypes.c_void_p
    lib.tilemix_route_words_per_row.argtypes = [P]
    lib.tilemix_route_words_per_row.restype = ctypes.c_int32
    lib.tilemix_workspace_size.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_workspace_size.restype = ctypes.c_int
    lib.tilemix_prefill.argtypes = [P, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_prefill.restype = ctypes.c_int
    lib.tilemix_fused_workspace_size.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_fused_workspace_size.restype = ctypes.c_int
    lib.tilemix_prefill_fused.argtypes = [P, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_prefill_fused.restype = ctypes.c_int
    lib.tilemix_prefill_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp]
    lib.tilemix_prefill_noalloc.restype = ctypes.c_int
    lib.tilemix_prepare.argtypes = [P, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_prepare.restype = ctypes.c_int
    lib.tilemix_attend.argtypes = [P, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_attend.restype = ctypes.c_int
    lib.tilemix_quantize.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    lib.tilemix_quantize.restype = ctypes.c_int
    lib.tilemix_debug_qk_int32.argtypes = [P, vp, vp, vp, ctypes.c_int32, vp, vp]
    lib.tilemix_debug_qk_int32.restype = ctypes.c_int
    TP = ctypes.POINTER(_CTemplate)
    lib.tilemix_auto_group_size.argtypes = [ctypes.c_int32, ctypes.c_int32]
    lib.tilemix_auto_group_size.restype = ctypes.c_int32
    lib.tilemix_route_template.argtypes = [P, TP, vp]
    lib.tilemix_route_template.restype = ctypes.c_int
    lib.tilemix_route_template_varlen.argtypes = [P, vp, vp, TP, vp]
    lib.tilemix_route_template_varlen.restype = ctypes.c_int
    lib.tilemix_varlen_workspace_size.argtypes = [P, ctypes.c_int32, ctypes.c_int32,
                                                  ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_varlen_workspace_size.restype = ctypes.c_int
    varlen_args = [P, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp,
                   ctypes.c_size_t, vp]
    lib.tilemix_prefill_varlen.argtypes = varlen_args
    lib.tilemix_prefill_varlen.restype = ctypes.c_int
    lib.tilemix_varlen_fused_workspace_size.argtypes = [P, ctypes.c_int32, ctypes.c_int32,
                                                        ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_varlen_fused_workspace_size.restype = ctypes.c_int
    lib.tilemix_prefill_varlen_fused.argtypes = varlen_args
    lib.tilemix_prefill_varlen_fused.restype = ctypes.c_int
    lib.tilemix_debug_prefill.argtypes = [P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp,
                                          vp, vp, vp, vp, ctypes.c_int32, vp, vp, ctypes.c_size_t,
                                          ctypes.POINTER(_CDebugExport), vp]
    lib.tilemix_debug_prefill.restype = ctypes.c_int
    lib.tilemix_quantize_kv.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    lib.tilemix_quantize_kv.restype = ctypes.c_int
    lib.tilemix_decode_workspace_size.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_decode_workspace_size.restype = ctypes.c_int
    lib.tilemix_decode.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_decode.restype = ctypes.c_int
    lib.tilemix_decode_varlen.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_decode_varlen.restype = ctypes.c_int
    CP = ctypes.c_char_p   # tilemix_paged_cache, packed into bytes (which may hold zeros: only its address counts)
    rows_args = [CP, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, vp]
    lib.tilemix_paged_append.argtypes = rows_args + [ctypes.c_int64, vp, ctypes.c_int64, vp]
    lib.tilemix_paged_append.restype = ctypes.c_int
    lib.tilemix_paged_gather.argtypes = rows_args + [vp, vp]
    lib.tilemix_paged_gather.restype = ctypes.c_int
    lib.tilemix_paged_decode_workspace_size.argtypes = [CP, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.tilemix_paged_decode_workspace_size.restype = ctypes.c_int
    lib.tilemix_paged_decode.argtypes = [CP, ctypes.c_int32, ctypes.c_int32, ctypes.c_float, ctypes.c_int32, vp,
                                         ctypes.c_int64, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tilemix_paged_decode.restype = ctypes.c_int
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.tilemix_paged_reserve.argtypes = [i32, i32, i32, vp, i64, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.tilemix_paged_reserve.restype = ctypes.c_int
    lib.tilemix_rotary_frequencies.argtypes = [CP, vp, ctypes.POINTER(ctypes.c_float)]
    lib.tilemix_rotary_frequencies.restype = ctypes.c_int
    lib.tilemix_rotary.argtypes = [CP, vp, vp, vp, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.tilemix_rotary.restype = ctypes.c_int
    lib.tilemix_route_coverage.argtypes = [P, vp, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_double)]
    lib.tilemix_route_coverage.restype = ctypes.c_int
    lib.tilemix_fit_template.argtypes = [P, TP, ctypes.c_double]
    lib.tilemix_fit_template.restype = ctypes.c_int
    lib.tilemix_status_string.argtypes = [ctypes.c_int]
    lib.tilemix_status_string.restype = ctypes.c_char_p
    lib.tilemix_last_error.argtypes = []
    lib.tilemix_last_error.restype = ctypes.c_char_p
    _LIB = lib
    return lib


def _check(status: int) -> None:
    if status != 0:
        lib = load_library()
        msg = lib.tilemix_last_error().decode() or lib.tilemix_status_string(status).decode()
        raise TilemixError(status, msg)


def _check_call(status: int) -> None:
    """_check for the calls that take a workspace: one that is too small is a ValueError."""
    if status == 5:
        raise ValueError(f"workspace too small: {load_library().tilemix_last_error().decode()}")
    if status != 0:
        _check(status)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    """The HIP stream as an integer (argtypes make it a void*).  The current one is asked for its
    handle directly: a torch.cuda.Stream object costs 2.5 us a call."""
    import torch
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _alloc(stream, *args, **kw):
    """torch.empty for a buffer the library uses on ``stream``: allocated while that stream is
    current, so that the caching allocator hands the block to no other stream's allocation
    before the work enqueued on ``stream`` is done with it."""
    torch = _torch()
    if stream is None:
        return torch.empty(*args, **kw)
    with torch.cuda.stream(stream):
        return torch.empty(*args, **kw)


def _alloc_like(stream, t, shape, dtype=None):
    """_alloc of a dense tensor on t's device, of t's type unless another is given.  (A call is a few microseconds, and
    these are the cheapest ways to a tensor.)"""
    if stream is None:
        if dtype is not None:
            return t.new_empty(shape, dtype=dtype)
        return _torch().empty_like(t) if t.shape == shape and t.is_contiguous() else t.new_empty(shape)
    return _alloc(stream, shape, dtype=t.dtype if dtype is None else dtype, device=t.device)


def tilemix_route_words_per_row(params: Params) -> int:
    return int(load_library().tilemix_route_words_per_row(ctypes.byref(params.c())))


def tilemix_workspace_size(params: Params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().tilemix_workspace_size(ctypes.byref(params.c()), ctypes.byref(n)))
    return int(n.value)


def _require(t, dtype, shape, name):
    import torch
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == shape
            and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint) -> _CParams:
    B, Lq, Hq, d = Q.shape
    Lk, Hk = K.shape[1], K.shape[2]
    return _cparams(B, Hq, Hk, Lq, Lk, d, tile, group_size, causal, scale, route_per_batch, route_hint)


def _check_inputs(cp: _CParams, Q, K, V=None):
    import torch
    kv = (cp.batch, cp.len_k, cp.heads_kv, cp.head_dim)
    _require(Q, torch.float16, (cp.batch, cp.len_q, cp.heads_q, cp.head_dim), "Q")
    _require(K, torch.float16, kv, "K")
    if V is not None:
        _require(V, torch.float16, kv, "V")


def _words_per_row(cp: _CParams) -> int:
    return load_library().tilemix_route_words_per_row(ctypes.byref(cp))


def _size(name: str, cp: _CParams, *args) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(load_library(), name)(ctypes.byref(cp), *args, ctypes.byref(n)))
    return n.value


def _workspace(workspace, device, stream, name: str, cp: _CParams, *args):
    """The caller's workspace (the library checks its size), or a new one of the size that the
    library's function ``name`` says."""
    if workspace is None:
        import torch
        need = _size(name, cp, *args)
        return _alloc(stream, need, dtype=torch.uint8, device=device), need
    return workspace, workspace.numel() * workspace.element_size()


def _route_and_out(cp: _CParams, Q, route_bits, O, stream=None):
    import torch
    T_m = -(-cp.len_q // cp.block_m) if cp.block_m > 0 else 0
    _require(route_bits, torch.int64,
             (cp.batch if cp.route_per_batch else 1, cp.heads_kv, T_m, _words_per_row(cp)), "route_bits")
    shape = (cp.batch, cp.len_q, cp.heads_q, cp.head_dim)
    if O is None:
        return _alloc(stream, shape, dtype=torch.float16, device=Q.device)
    _require(O, torch.float16, shape, "O")
    return O


def _prefill_call(name, size, Q, K, V, route_bits, group_size, tile, causal, scale, O, workspace, stream,
                  route_per_batch, route_hint):
    cp = _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint)
    _check_inputs(cp, Q, K, V)
    O = _route_and_out(cp, Q, route_bits, O, stream)
    workspace, nbytes = _workspace(workspace, Q.device, stream, size, cp)
    _check_call(getattr(load_library(), name)(
        ctypes.byref(cp), Q.data_ptr(), K.data_ptr(), V.data_ptr(), route_bits.data_ptr(), O.data_ptr(),
        workspace.data_ptr(), nbytes, _stream(stream)))
    return O


def tilemix_prefill(Q, K, V, route_bits, group_size: int, tile=(128, 64), causal: bool = True,
                    scale: float | None = None, *, O=None, workspace=None, stream=None,
                    route_per_batch: bool = False, route_hint: int = -1):
    """Routed prefill attention.  Q [B, Lq, Hq, d], K/V [B, Lk, Hk, d] fp16 CUDA tensors,
    route_bits uint64 words [B_r, Hk, T_m, W] as an int64 CUDA tensor (same bits).
    Returns O (fp16, [B, Lq, Hq, d]).  ``workspace`` (uint8, >= tilemix_workspace_size)
    is allocated when not given."""
    return _prefill_call("tilemix_prefill", "tilemix_workspace_size", Q, K, V, route_bits, group_size, tile,
                         causal, scale, O, workspace, stream, route_per_batch, route_hint)


def tilemix_fused_workspace_size(params: Params) -> int:
    n = ctypes.c_size_t()
    _check(load_library().tilemix_fused_workspace_size(ctypes.byref(params.c()), ctypes.byref(n)))
    return n.value


def tilemix_prefill_fused(Q, K, V, route_bits, group_size: int, tile=(128, 64), causal: bool = True,
                          scale: float | None = None, *, O=None, workspace=None, stream=None,
                          route_per_batch: bool = False, route_hint: int = -1):
    """Routed prefill attention in the fused on-the-fly operand mode (no Q8/K8 scratch; the
    kernel quantizes on chip).  Arguments and result as tilemix_prefill; ``workspace`` (uint8,
    >= tilemix_fused_workspace_size) is allocated when not given."""
    return _prefill_call("tilemix_prefill_fused", "tilemix_fused_workspace_size", Q, K, V, route_bits,
                         group_size, tile, causal, scale, O, workspace, stream, route_per_batch, route_hint)


NOALLOC_SCRATCH_BYTES = 128 << 20   # TILEMIX_NOALLOC_SCRATCH_BYTES


def tilemix_prefill_noalloc(Q, K, V, route_bits, group_size: int, tile=(128, 64),
                            causal: bool = True, scale: float | None = None, *, O, stream=None,
                            route_per_batch: bool = False, route_hint: int = -1):
    """tilemix_prefill with no allocation and no workspace argument: the library serves the
    workspace from its own per-GPU device array (at most NOALLOC_SCRATCH_BYTES).  ``O`` is
    required; nothing is allocated here either.  Calls that overlap on one GPU race."""
    cp = _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint)
    _check_inputs(cp, Q, K, V)
    O = _route_and_out(cp, Q, route_bits, O, stream)
    _check(load_library().tilemix_prefill_noalloc(
        ctypes.byref(cp), Q.data_ptr(), K.data_ptr(), V.data_ptr(), route_bits.data_ptr(), O.data_ptr(),
        _stream(stream)))
    return O


def tilemix_prepare(Q, K, V, group_size: int, tile=(128, 64), causal: bool = True,
                    scale: float | None = None, *, workspace=None, stream=None,
                    route_per_batch: bool = False, route_hint: int = -1):
    """Operand preparation (quantize-once + V tile layout) into ``workspace``; returns it."""
    cp = _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint)
    _check_inputs(cp, Q, K, V)
    workspace, nbytes = _workspace(workspace, Q.device, stream, "tilemix_workspace_size", cp)
    _check_call(load_library().tilemix_prepare(ctypes.byref(cp), Q.data_ptr(), K.data_ptr(), V.data_ptr(),
                                               workspace.data_ptr(), nbytes, _stream(stream)))
    return workspace


def tilemix_attend(Q, K, route_bits, workspace, group_size: int, tile=(128, 64), causal: bool = True,
                   scale: float | None = None, *, O=None, stream=None, route_per_batch: bool = False,
                   route_hint: int = -1):
    """Fused routed attention on a workspace filled by tilemix_prepare; returns O."""
    cp = _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint)
    _check_inputs(cp, Q, K)
    O = _route_and_out(cp, Q, route_bits, O, stream)
    workspace, nbytes = _workspace(workspace, Q.device, stream, "tilemix_workspace_size", cp)
    _check_call(load_library().tilemix_attend(ctypes.byref(cp), Q.data_ptr(), K.data_ptr(), route_bits.data_ptr(),
                                              O.data_ptr(), workspace.data_ptr(), nbytes, _stream(stream)))
    return O


def tilemix_quantize(Q, K, *, tile=(128, 64), stream=None):
    """Quantize-once pass.  Returns (Q8 int8, dQ fp16, K8 int8, dK fp16) CUDA tensors."""
    import torch
    B, Lq, Hq, d = Q.shape
    Lk, Hk = K.shape[1], K.shape[2]
    p = Params(B, Hq, Hk, Lq, Lk, d, tile[0], tile[1])
    _require(Q, torch.float16, (B, Lq, Hq, d), "Q")
    _require(K, torch.float16, (B, Lk, Hk, d), "K")
    Q8 = _alloc(stream, (B, Lq, Hq, d), dtype=torch.int8, device=Q.device)
    K8 = _alloc(stream, (B, Lk, Hk, d), dtype=torch.int8, device=Q.device)
    dQ = _alloc(stream, (B, -(-Lq // 128), Hq), dtype=torch.float16, device=Q.device)
    dK = _alloc(stream, (B, -(-Lk // 64), Hk), dtype=torch.float16, device=Q.device)
    cp = p.c()
    _check(load_library().tilemix_quantize(ctypes.byref(cp), Q.data_ptr(), K.data_ptr(), Q8.data_ptr(),
                                           dQ.data_ptr(), K8.data_ptr(), dK.data_ptr(), _stream(stream)))
    return Q8, dQ, K8, dK


def tilemix_debug_qk_int32(Q8, K8, tiles, *, heads_q: int, heads_kv: int, tile=(128, 64),
                           stream=None):
    """INT32 tile products for rows (b, h_q, m, n) of ``tiles`` (int32 CUDA [count, 4]).
    Returns int32 [count, BLOCK_M, BLOCK_N]."""
    import torch
    B, Lq, Hq, d = Q8.shape
    Lk = K8.shape[1]
    p = Params(B, heads_q, heads_kv, Lq, Lk, d, tile[0], tile[1])
    _require(Q8, torch.int8, (B, Lq, heads_q, d), "Q8")
    _require(K8, torch.int8, (B, Lk, heads_kv, d), "K8")
    count = tiles.shape[0]
    _require(tiles, torch.int32, (count, 4), "tiles")
    out = _alloc(stream, (count, tile[0], tile[1]), dtype=torch.int32, device=Q8.device)
    cp = p.c()
    _check(load_library().tilemix_debug_qk_int32(ctypes.byref(cp), _ptr(Q8), _ptr(K8), _ptr(tiles),
                                                 ctypes.c_int32(count), _ptr(out), _stream(stream)))
    return out


# ----------------------------------------------------------------- routing templates (host)

def tilemix_auto_group_size(len_k: int, block_n: int = 64) -> int:
    """The paper's automatic routing-group size g for L_k keys (0 if an argument is < 1)."""
    return int(load_library().tilemix_auto_group_size(len_k, block_n))


def _host_words_shape(p: Params):
    return (p.batch if p.route_per_batch else 1, p.heads_kv, p.T_m, tilemix_route_words_per_row(p))


def tilemix_route_template(params: Params, template: Template):
    """Routing words (host NumPy uint64 [B_r, H_k, T_m, W]) of ``template`` for ``params``."""
    import numpy as np
    shape = _host_words_shape(params)
    words = np.zeros(shape, dtype=np.uint64)
    cp, ct = params.c(), template.c()
    _check(load_library().tilemix_route_template(ctypes.byref(cp), ctypes.byref(ct),
                                                 words.ctypes.data_as(ctypes.c_void_p)))
    return words


def tilemix_route_coverage(params: Params, words):
    """(rho_groups, rho_pairs): realized INT8 coverage of host routing words."""
    import numpy as np
    w = np.ascontiguousarray(words, dtype=np.uint64)
    if w.shape != _host_words_shape(params):
        raise ValueError(f"words must have shape {_host_words_shape(params)}, got {w.shape}")
    rg, rp = ctypes.c_double(0.0), ctypes.c_double(0.0)
    cp = params.c()
    _check(load_library().tilemix_route_coverage(ctypes.byref(cp), w.ctypes.data_as(ctypes.c_void_p),
                                                 ctypes.byref(rg), ctypes.byref(rp)))
    return rg.value, rp.value


def tilemix_fit_template(params: Params, template: Template, rho_int8: float) -> Template:
    """The template with its size parameter chosen to match INT8 coverage ``rho_int8``."""
    cp, ct = params.c(), template.c()
    _check(load_library().tilemix_fit_template(ctypes.byref(cp), ctypes.byref(ct),
                                               ctypes.c_double(rho_int8)))
    return Template.from_c(template.kind, ct)


def tilemix_route_template_varlen(params: Params, seqlens_q, seqlens_k, template: Template):
    """Routing words (host uint64 [sum_b ceil(L_q,b / BLOCK_M), H_k, W]) of ``template`` for each
    sequence of a variable-length batch (``params.len_q``/``len_k`` = maximum lengths)."""
    import numpy as np
    lq = np.ascontiguousarray(seqlens_q, dtype=np.int32)
    lk = np.ascontiguousarray(seqlens_k, dtype=np.int32)
    if lq.shape != (params.batch,) or lk.shape != (params.batch,):
        raise ValueError("seqlens_q / seqlens_k must have one entry per sequence")
    rows = int(sum(-(-int(x) // params.block_m) for x in lq))
    words = np.zeros((rows, params.heads_kv, tilemix_route_words_per_row(params)), dtype=np.uint64)
    cp, ct = params.c(), template.c()
    _check(load_library().tilemix_route_template_varlen(
        ctypes.byref(cp), lq.ctypes.data_as(ctypes.c_void_p), lk.ctypes.data_as(ctypes.c_void_p),
        ctypes.byref(ct), words.ctypes.data_as(ctypes.c_void_p)))
    return words


def tilemix_varlen_workspace_size(params: Params, total_q: int, total_k: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().tilemix_varlen_workspace_size(ctypes.byref(params.c()), total_q, total_k,
                                                        ctypes.byref(n)))
    return int(n.value)


def tilemix_varlen_fused_workspace_size(params: Params, total_q: int, total_k: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().tilemix_varlen_fused_workspace_size(ctypes.byref(params.c()), total_q,
                                                              total_k, ctypes.byref(n)))
    return int(n.value)


def _varlen_call(name, Q, K, V, cu_seqlens_q, cu_seqlens_k, max_len_q, max_len_k, route_bits,
                 group_size, tile, causal, scale, O, workspace, stream, route_hint, fused):
    import torch
    total_q, Hq, d = Q.shape
    total_k, Hk = K.shape[0], K.shape[1]
    B = cu_seqlens_q.shape[0] - 1
    cp = _cparams(B, Hq, Hk, max_len_q, max_len_k, d, tile, group_size, causal, scale, False, route_hint)
    _require(Q, torch.float16, (total_q, Hq, d), "Q")
    _require(K, torch.float16, (total_k, Hk, d), "K")
    _require(V, torch.float16, (total_k, Hk, d), "V")
    _require(cu_seqlens_q, torch.int32, (B + 1,), "cu_seqlens_q")
    _require(cu_seqlens_k, torch.int32, (B + 1,), "cu_seqlens_k")
    if route_bits.dim() != 3 or tuple(route_bits.shape[1:]) != (Hk, _words_per_row(cp)):
        raise ValueError("route_bits must be [rows, H_k, W]")
    _require(route_bits, torch.int64, tuple(route_bits.shape), "route_bits")
    if O is None:
        O = _alloc(stream, (total_q, Hq, d), dtype=torch.float16, device=Q.device)
    _require(O, torch.float16, (total_q, Hq, d), "O")
    size = "tilemix_varlen_fused_workspace_size" if fused else "tilemix_varlen_workspace_size"
    workspace, nbytes = _workspace(workspace, Q.device, stream, size, cp, total_q, total_k)
    _check_call(getattr(load_library(), name)(
        ctypes.byref(cp), total_q, total_k, cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), Q.data_ptr(),
        K.data_ptr(), V.data_ptr(), route_bits.data_ptr(), route_bits.shape[0], O.data_ptr(),
        workspace.data_ptr(), nbytes, _stream(stream)))
    return O


def tilemix_prefill_varlen(Q, K, V, cu_seqlens_q, cu_seqlens_k, max_len_q: int, max_len_k: int,
                           route_bits, group_size: int, tile=(128, 64), causal: bool = True,
                           scale: float | None = None, *, O=None, workspace=None, stream=None,
                           route_hint: int = -1):
    """Routed prefill attention over a packed variable-length batch.  Q [total_q, Hq, d],
    K/V [total_k, Hk, d] fp16 CUDA tensors; cu_seqlens_q/k int32 CUDA [B + 1]; route_bits the
    uint64 words [sum_b ceil(L_q,b / BLOCK_M), Hk, W] as an int64 CUDA tensor.  Returns O."""
    return _varlen_call("tilemix_prefill_varlen", Q, K, V, cu_seqlens_q, cu_seqlens_k, max_len_q,
                        max_len_k, route_bits, group_size, tile, causal, scale, O, workspace, stream,
                        route_hint, False)


def tilemix_prefill_varlen_fused(Q, K, V, cu_seqlens_q, cu_seqlens_k, max_len_q: int,
                                 max_len_k: int, route_bits, group_size: int, tile=(128, 64),
                                 causal: bool = True, scale: float | None = None, *, O=None,
                                 workspace=None, stream=None, route_hint: int = -1):
    """tilemix_prefill_varlen in the fused on-the-fly operand mode (no K8 / scale tensors)."""
    return _varlen_call("tilemix_prefill_varlen_fused", Q, K, V, cu_seqlens_q, cu_seqlens_k,
                        max_len_q, max_len_k, route_bits, group_size, tile, causal, scale, O,
                        workspace, stream, route_hint, True)


def tilemix_debug_prefill(Q, K, V, route_bits, group_size: int, tile=(128, 64), causal: bool = True,
                          scale: float | None = None, *, fused: bool = False, cu_seqlens_q=None,
                          cu_seqlens_k=None, max_len_q: int = 0, max_len_k: int = 0,
                          route_per_batch: bool = False, route_hint: int = -1, stream=None):
    """Test entry point: one prefill call (fixed-length [B, L, H, d] inputs, or packed
    [total, H, d] ones with ``cu_seqlens_q/k`` and the maximum lengths) whose kernel also exports
    the INT8 operands it made and multiplied.  Returns (O, q8, dq, tiles, kinds): q8 like Q
    (pre-filled with -128), dq int16 bits [R, Hq] (pre-filled with -1), tiles int32
    [R, Hq, T_n, BLOCK_M, 64] and kinds int32 [R, Hq, T_n, BLOCK_M // 32] (pre-filled with 0),
    R the query-tile rows (B * T_m, or the rows of ``route_bits`` for a packed batch)."""
    import torch
    varlen = cu_seqlens_q is not None
    if varlen:
        total_q, Hq, d = Q.shape
        total_k, Hk = K.shape[0], K.shape[1]
        B = cu_seqlens_q.shape[0] - 1
        p = Params(B, Hq, Hk, max_len_q, max_len_k, d, tile[0], tile[1], group_size, causal,
                   scale if scale else 1.0 / math.sqrt(d), False, route_hint)
        cp = p.c()
        _require(Q, torch.float16, (total_q, Hq, d), "Q")
        _require(K, torch.float16, (total_k, Hk, d), "K")
        _require(V, torch.float16, (total_k, Hk, d), "V")
        _require(cu_seqlens_q, torch.int32, (B + 1,), "cu_seqlens_q")
        _require(cu_seqlens_k, torch.int32, (B + 1,), "cu_seqlens_k")
        if route_bits.dim() != 3 or tuple(route_bits.shape[1:]) != (Hk, tilemix_route_words_per_row(p)):
            raise ValueError("route_bits must be [rows, H_k, W]")
        _require(route_bits, torch.int64, tuple(route_bits.shape), "route_bits")
        rows = route_bits.shape[0]
        O = _alloc(stream, (total_q, Hq, d), dtype=torch.float16, device=Q.device)
        size = "tilemix_varlen_fused_workspace_size" if fused else "tilemix_varlen_workspace_size"
        size_args = (total_q, total_k)
    else:
        cp = _prefill_params(Q, K, group_size, tile, causal, scale, route_per_batch, route_hint)
        _check_inputs(cp, Q, K, V)
        O = _route_and_out(cp, Q, route_bits, None, stream)
        p = Params(cp.batch, cp.heads_q, cp.heads_kv, cp.len_q, cp.len_k, cp.head_dim, tile[0], tile[1])
        total_q = total_k = -1
        rows = p.batch * p.T_m
        size = "tilemix_fused_workspace_size" if fused else "tilemix_workspace_size"
        size_args = ()
    workspace, nbytes = _workspace(None, Q.device, stream, size, cp, *size_args)
    q8 = _alloc(stream, tuple(Q.shape), dtype=torch.int8, device=Q.device)
    dq = _alloc(stream, (rows, p.heads_q), dtype=torch.int16, device=Q.device)
    tiles = _alloc(stream, (rows, p.heads_q, p.T_n, p.block_m, 64), dtype=torch.int32, device=Q.device)
    kinds = _alloc(stream, (rows, p.heads_q, p.T_n, p.block_m // 32), dtype=torch.int32,
                   device=Q.device)
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        q8.fill_(-128)
        dq.fill_(-1)
        tiles.zero_()
        kinds.zero_()
    exp = _CDebugExport(_ptr(q8), _ptr(dq), _ptr(tiles), _ptr(kinds))
    _check(load_library().tilemix_debug_prefill(
        ctypes.byref(cp), int(bool(fused)), total_q, total_k, _ptr(cu_seqlens_q), _ptr(cu_seqlens_k),
        _ptr(Q), _ptr(K), _ptr(V), _ptr(route_bits), ctypes.c_int32(rows if varlen else 0), _ptr(O),
        _ptr(workspace), ctypes.c_size_t(nbytes), ctypes.byref(exp), _stream(stream)))
    return O, q8, dq, tiles, kinds


# ------------------------------------------------------------ INT8 key/value cache decode

def tilemix_quantize_kv(K, V, *, stream=None):
    """INT8 key/value cache of K, V [B, L_k, H_k, d] (fp16 CUDA): (K8, dK, V8, dV) with K8
    [B, L_k, H_k, d] and V8 [B, H_k, ceil(L_k/64), d, 64] (each 64-key block channel-major)."""
    import torch
    B, Lk, Hk, d = K.shape
    cp = _cparams(B, Hk, Hk, 1, Lk, d, (128, 64), 1, True, None, False, -1)
    _require(K, torch.float16, (B, Lk, Hk, d), "K")
    _require(V, torch.float16, (B, Lk, Hk, d), "V")
    K8 = _alloc(stream, (B, Lk, Hk, d), dtype=torch.int8, device=K.device)
    V8 = _alloc(stream, (B, Hk, -(-Lk // 64), d, 64), dtype=torch.int8, device=K.device)
    dK = _alloc(stream, (B, -(-Lk // 64), Hk), dtype=torch.float16, device=K.device)
    dV = _alloc(stream, (B, -(-Lk // 64), Hk), dtype=torch.float16, device=K.device)
    _check(load_library().tilemix_quantize_kv(ctypes.byref(cp), K.data_ptr(), V.data_ptr(), K8.data_ptr(),
                                              dK.data_ptr(), V8.data_ptr(), dV.data_ptr(), _stream(stream)))
    return K8, dK, V8, dV


def tilemix_decode_workspace_size(params: Params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().tilemix_decode_workspace_size(ctypes.byref(params.c()), ctypes.byref(n)))
    return int(n.value)


def tilemix_decode(Q, K, K8, dK, V8, dV, route_bits, group_size: int, scale: float | None = None,
                   *, O=None, workspace=None, stream=None, route_per_batch: bool = False,
                   route_hint: int = -1, seqlens_k=None):
    """One decode step: Q [B, 1, Hq, d] against the FP16 key cache K [B, L_k, H_k, d] and the
    INT8 caches of tilemix_quantize_kv; route_bits int64 CUDA [B_r, H_k, 1, W].  Returns O.
    With ``seqlens_k`` (int32 CUDA [B]) sequence b uses its first seqlens_k[b] cached keys
    (tilemix_decode_varlen; L_k is then the caches' capacity)."""
    import torch
    B, Lq, Hq, d = Q.shape
    Lk, Hk = K.shape[1], K.shape[2]
    cp = _cparams(B, Hq, Hk, Lq, Lk, d, (128, 64), group_size, True, scale, route_per_batch, route_hint)
    _require(Q, torch.float16, (B, 1, Hq, d), "Q")
    _require(K, torch.float16, (B, Lk, Hk, d), "K")
    _require(K8, torch.int8, (B, Lk, Hk, d), "K8")
    _require(V8, torch.int8, (B, Hk, -(-Lk // 64), d, 64), "V8")
    _require(dK, torch.float16, (B, -(-Lk // 64), Hk), "dK")
    _require(dV, torch.float16, (B, -(-Lk // 64), Hk), "dV")
    _require(route_bits, torch.int64, (B if route_per_batch else 1, Hk, 1, _words_per_row(cp)),
             "route_bits")
    if O is None:
        O = _alloc(stream, tuple(Q.shape), dtype=torch.float16, device=Q.device)
    else:
        _require(O, torch.float16, (B, 1, Hq, d), "O")
    workspace, nbytes = _workspace(workspace, Q.device, stream, "tilemix_decode_workspace_size", cp)
    rest = (Q.data_ptr(), K.data_ptr(), K8.data_ptr(), dK.data_ptr(), V8.data_ptr(), dV.data_ptr(),
            route_bits.data_ptr(), O.data_ptr(), workspace.data_ptr(), nbytes, _stream(stream))
    if seqlens_k is not None:
        _require(seqlens_k, torch.int32, (B,), "seqlens_k")
        _check_call(load_library().tilemix_decode_varlen(ctypes.byref(cp), seqlens_k.data_ptr(), *rest))
    else:
        _check_call(load_library().tilemix_decode(ctypes.byref(cp), *rest))
    return O


# -------------------------------------------------------------------- paged key/value cache

class PagedCache(NamedTuple):
    """A pool of pages for ``tilemix_paged_append``, ``_gather`` and ``_decode``: K, V [P, Hk, page, d] CUDA
    tensors in float16, bfloat16, int8 or float8_e4m3fn, and for the last two dK, dV float32
    [P, Hk, page], one scale per row; or, in 4 bits, K, V float4_e2m1fn_x2 [P, Hk, page, d / 2] (two
    channels to an element, the even one in the low bits) and dK, dV float8_e8m0fnu [P, Hk, page, d / 32],
    a power of two for each 32 channels.  Each page is dense; pages may lie further apart (a slice of a
    larger tensor).  A page holds 16, 32, 64, 128 or 256 tokens, d is 64 or 128."""
    K: object
    V: object
    dK: object = None
    dV: object = None

    @staticmethod
    def empty(pages: int, page_size: int, heads_kv: int, head_dim: int, dtype=None, device="cuda") -> "PagedCache":
        """An uninitialised pool (int8 when no dtype is given)."""
        torch = _torch()
        dtype = torch.int8 if dtype is None else dtype
        shape = (pages, heads_kv, page_size, head_dim)
        if _format(dtype) == 5:
            return PagedCache(*(torch.empty((*shape[:3], head_dim // n), dtype=t, device=device)
                                for n, t in ((2, dtype), (2, dtype), (32, torch.float8_e8m0fnu), (32, torch.float8_e8m0fnu))))
        K, V = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        if dtype.itemsize == 2:
            return PagedCache(K, V)
        dK, dV = (torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2))
        return PagedCache(K, V, dK, dV)


# tilemix_paged_cache: format, pages, page_size, heads_kv, head_dim, batch, max_pages; stride_k, _v, _dk, _dv,
# _table; K, V, dK, dV, page_table, seqlens_k.  Packed in one go: a decode step is a few microseconds.
_PAGED = struct.Struct("<7i4x5q6Q")
_FORMATS: dict = {}
_TORCH = None


def _torch():
    """torch, imported once (an import statement costs 0.3 us each time it is met)."""
    global _TORCH
    if _TORCH is None:
        import torch
        _FORMATS.update({torch.float16: 0, torch.bfloat16: 1, torch.int8: 2, torch.float8_e4m3fn: 3})
        if hasattr(torch, "float4_e2m1fn_x2"):   # (without the type there are no pools of it, and all else works)
            _FORMATS[torch.float4_e2m1fn_x2] = 5
        _TORCH = torch
    return _TORCH


def _format(dtype) -> int:
    """tilemix_format of a torch dtype, or -1."""
    return _FORMATS.get(dtype, -1)


def _require_like(t, dtype, shape, device, name):
    """A CUDA tensor of this type and shape on this device (an index)."""
    try:
        if t.dtype == dtype and t.shape == shape and t.get_device() == device:
            return
    except AttributeError:
        pass
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be on the pool's device")


def _require_dense(t, dtype, shape, device, name):
    _require_like(t, dtype, shape, device, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _outer_stride(shape, stride, dims: int, name: str) -> int:
    """Elements between the entries of the dimension before the last ``dims``, which must be dense (the stride
    of a dimension of size 1 means nothing)."""
    inner = 1
    for i in range(1, dims + 1):
        if shape[-i] != 1 and stride[-i] != inner:
            raise ValueError(f"{name}: the last {dims} dimensions must be dense")
        inner *= shape[-i]
    return inner if shape[-dims - 1] == 1 else stride[-dims - 1]


def _paged(cache: PagedCache, page_table, seqlens_k):
    """(tilemix_paged_cache as bytes, format, device index, B, Hk, d)."""
    torch = _torch()
    K, V, dK, dV = cache
    if not isinstance(K, torch.Tensor) or not K.is_cuda:
        raise TypeError("the pool's K must be a CUDA (HIP) tensor")
    dtype, shape, dev = K.dtype, K.shape, K.get_device()
    fmt = _format(dtype)
    if fmt < 0:
        raise TypeError(f"the pool must be float16, bfloat16, int8, float8_e4m3fn or float4_e2m1fn_x2, got {dtype}")
    if len(shape) != 4:
        raise ValueError(f"the pool's K must be [pages, Hk, page, d], got {tuple(shape)}")
    _require_like(V, dtype, shape, dev, "the pool's V")
    P, Hk, page, d = shape
    per = Hk * page
    # (What is contiguous, as it mostly is, needs no look at its strides.)
    sk = per * d if K.is_contiguous() else _outer_stride(shape, K.stride(), 3, "the pool's K")
    sv = per * d if V.is_contiguous() else _outer_stride(shape, V.stride(), 3, "the pool's V")
    sdk = sdv = pdk = pdv = 0
    if fmt >= 2:
        if fmt == 5:
            if d % 16:   # (where this is refused, the message speaks of d)
                raise ValueError(f"head_dim {2 * d} not supported (64 or 128)")
            rows, of, inner = (P, Hk, page, d // 16), torch.float8_e8m0fnu, 3
            per *= d // 16
            d *= 2
        else:
            rows, of, inner = shape[:3], torch.float32, 2
        _require_like(dK, of, rows, dev, "the pool's dK")
        _require_like(dV, of, rows, dev, "the pool's dV")
        sdk = per if dK.is_contiguous() else _outer_stride(rows, dK.stride(), inner, "the pool's dK")
        sdv = per if dV.is_contiguous() else _outer_stride(rows, dV.stride(), inner, "the pool's dV")
        pdk, pdv = dK.data_ptr(), dV.data_ptr()
    if getattr(page_table, "ndim", None) != 2:
        raise ValueError("page_table must be a tensor [B, max_pages]")
    t_shape = page_table.shape
    _require_like(page_table, torch.int32, t_shape, dev, "page_table")
    B, entries = t_shape
    _require_dense(seqlens_k, torch.int32, (B,), dev, "seqlens_k")
    return _PAGED.pack(fmt, P, page, Hk, d, B, entries, sk, sv, sdk, sdv,
                       entries if page_table.is_contiguous() else _outer_stride(t_shape, page_table.stride(), 1, "page_table"),
                       K.data_ptr(), V.data_ptr(), pdk, pdv, page_table.data_ptr(), seqlens_k.data_ptr()), fmt, dev, B, Hk, d


def _int32(n: int, name: str) -> int:
    """n, which ctypes would take modulo 2^32."""
    if -0x80000000 <= n < 0x80000000:
        return n
    raise ValueError(f"{name} ({n}) does not fit in 32 bits")


def _paged_rows(cu_seqlens, max_len, total, device, B, Hk, d):
    """(cu_seqlens pointer, total, shape of the rows) of an append or gather."""
    _int32(max_len, "max_len")
    if cu_seqlens is None:
        return None, _int32(B * max_len, "B * max_len"), (B, max_len, Hk, d)
    _int32(total, "total")
    _require_dense(cu_seqlens, _torch().int32, (B + 1,), device, "cu_seqlens")
    return cu_seqlens.data_ptr(), total, (total, Hk, d)


def _row_stride(t, shape, name: str) -> int:
    """Elements between the token rows of t, [total, Hk, d] or [B, len, Hk, d]."""
    if t.is_contiguous():
        return shape[-2] * shape[-1]
    stride = t.stride()
    if len(shape) == 3:
        return _outer_stride(shape, stride, 2, name)
    B, L, Hk, d = shape
    if L == 1:   # one row per sequence: they are as far apart as the sequences
        return _outer_stride((B, Hk, d), (stride[0], stride[2], stride[3]), 2, name)
    row = _outer_stride(shape, stride, 2, name)
    if B > 1 and L > 1 and stride[0] != L * row:
        raise ValueError(f"{name}: the rows of all sequences must be equally far apart")
    return row


def _stream_on(stream, device: int) -> int:
    """The HIP stream as an integer: ``stream``, or the device's current one."""
    if stream is None:
        return _torch()._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise ValueError("stream must be on the pool's device")
    return stream.cuda_stream


def _elsewhere(device: int):
    """The library launches on the current device.  None where that is the tensors' own, or a context in which
    it is: the caller then calls itself again in it."""
    torch = _torch()
    return None if torch._C._cuda_getDevice() == device else torch.cuda.device(device)


def tilemix_paged_append(cache: PagedCache, K, V, page_table, seqlens_k, cu_seqlens=None,
                         max_len: int | None = None, *, stream=None) -> None:
    """Write new rows into a paged cache; they are the last rows of their sequences, which
    ``seqlens_k`` (int32 CUDA [B]) counts already.  K, V: float16 or bfloat16 CUDA [total, Hk, d] with
    ``cu_seqlens`` (int32 CUDA [B + 1]) and ``max_len`` >= the most rows of a sequence, or
    [B, L, Hk, d], L rows for each sequence (1: a decode step).  Tokens may lie any multiple of 8 elements
    apart.  page_table: int32 CUDA [B, max_pages]; ids outside the pool name no page."""
    c, _, dev, B, Hk, d = _paged(cache, page_table, seqlens_k)
    packed = cu_seqlens is not None
    if getattr(K, "ndim", None) != (3 if packed else 4):
        raise ValueError("K and V must be [total, Hk, d] with cu_seqlens, and [B, L, Hk, d] without")
    if packed:
        if max_len is None:
            raise ValueError("max_len is needed with cu_seqlens")
    elif max_len is None:
        max_len = K.shape[1]
    elif max_len != K.shape[1]:
        raise ValueError("max_len is the rows of K without cu_seqlens")
    cu, total, shape = _paged_rows(cu_seqlens, max_len, K.shape[0], dev, B, Hk, d)
    dtype = K.dtype
    fmt = _format(dtype)
    if fmt not in (0, 1):
        raise TypeError(f"K must be float16 or bfloat16, got {dtype}")
    _require_like(K, dtype, shape, dev, "K")
    _require_like(V, dtype, shape, dev, "V")
    other = _elsewhere(dev)
    if other is not None:
        with other:
            return tilemix_paged_append(cache, K, V, page_table, seqlens_k, cu_seqlens, max_len, stream=stream)
    _check(load_library().tilemix_paged_append(c, fmt, cu, max_len, total, K.data_ptr(), _row_stride(K, shape, "K"),
                                               V.data_ptr(), _row_stride(V, shape, "V"), _stream_on(stream, dev)))


def tilemix_paged_gather(cache: PagedCache, page_table, seqlens_k, max_len: int, cu_seqlens=None,
                         total: int | None = None, *, dtype=None, K=None, V=None, stream=None):
    """Read the last rows of every sequence back: with ``cu_seqlens`` (int32 CUDA [B + 1]) sequence b's last
    cu_seqlens[b + 1] - cu_seqlens[b] rows, packed [total, Hk, d], none with more than ``max_len``; else
    its last max_len rows, [B, max_len, Hk, d].  Returns (K, V) in ``dtype`` (that of a 16-bit pool;
    float16 by default for the others), written into ``K`` and ``V`` if given; float16 ones are the K and V of
    tilemix_prefill_varlen (which takes no bfloat16).  Tokens that the cache does not hold are zeros; packed rows
    that no sequence owns are not written."""
    torch = _torch()
    c, pool, dev, B, Hk, d = _paged(cache, page_table, seqlens_k)
    if dtype is None:
        dtype = K.dtype if K is not None else cache.K.dtype if pool < 2 else torch.float16
    fmt = _format(dtype)
    if fmt not in (0, 1):
        raise TypeError(f"dtype must be float16 or bfloat16, got {dtype}")
    if cu_seqlens is not None and total is None:
        if K is None:
            raise ValueError("total is needed with cu_seqlens")
        total = K.shape[0]
    if cu_seqlens is None and total not in (None, B * max_len):
        raise ValueError("total is B * max_len without cu_seqlens")
    rows, total, shape = _paged_rows(cu_seqlens, max_len, total, dev, B, Hk, d)
    other = _elsewhere(dev)
    if other is not None:
        with other:
            return tilemix_paged_gather(cache, page_table, seqlens_k, max_len, cu_seqlens, total, dtype=dtype, K=K, V=V,
                                        stream=stream)
    handle = _stream_on(stream, dev)
    if K is None:
        K = _alloc_like(stream, cache.K, shape, dtype)
    else:
        _require_dense(K, dtype, shape, dev, "K")
    if V is None:
        V = _alloc_like(stream, K, shape)
    else:
        _require_dense(V, dtype, shape, dev, "V")
    _check(load_library().tilemix_paged_gather(c, fmt, rows, max_len, total, K.data_ptr(), V.data_ptr(), handle))
    return K, V


def tilemix_paged_decode_workspace_size(cache: PagedCache, page_table, seqlens_k, heads_q: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().tilemix_paged_decode_workspace_size(_paged(cache, page_table, seqlens_k)[0], _int32(heads_q, "heads_q"),
                                                              ctypes.byref(n)))
    return n.value


def tilemix_paged_decode(cache: PagedCache, Q, page_table, seqlens_k, scale: float | None = None, *, window: int = 0,
                         O=None, lse=None, return_lse: bool = False, workspace=None, stream=None):
    """One decode step over a paged cache: Q [B, 1, Hq, d] (float16 or bfloat16, that of a 16-bit pool; sequences
    may lie any multiple of 8 elements apart) attends to each sequence's ``seqlens_k`` tokens, or its
    last ``window`` >= 1.  Returns O, like Q, and with ``return_lse`` (O, lse): float32 [B, Hq], the log of
    the sum of e^score.  A sequence without a token gets O = 0 and lse = -inf.  ``O``, ``lse`` and ``workspace``
    (uint8, >= tilemix_paged_decode_workspace_size) are allocated when not given."""
    torch = _torch()
    c, _, dev, B, Hk, d = _paged(cache, page_table, seqlens_k)
    if getattr(Q, "ndim", None) != 4:
        raise ValueError("Q must be [B, 1, Hq, d]")
    dtype = Q.dtype
    fmt = _format(dtype)
    if fmt not in (0, 1):
        raise TypeError(f"Q must be float16 or bfloat16, got {dtype}")
    heads = Q.shape[2]
    shape = (B, 1, heads, d)
    _require_like(Q, dtype, shape, dev, "Q")
    q_stride = _row_stride(Q, shape, "Q")
    _int32(window, "window")
    other = _elsewhere(dev)
    if other is not None:
        with other:
            return tilemix_paged_decode(cache, Q, page_table, seqlens_k, scale, window=window, O=O, lse=lse,
                                        return_lse=return_lse, workspace=workspace, stream=stream)
    handle, lib = _stream_on(stream, dev), load_library()
    if O is None:
        O = _alloc_like(stream, Q, shape)
    else:
        _require_dense(O, dtype, shape, dev, "O")
    if lse is not None:
        _require_dense(lse, torch.float32, (B, heads), dev, "lse")
    elif return_lse:
        lse = _alloc_like(stream, Q, (B, heads), torch.float32)
    if workspace is None:
        n = ctypes.c_size_t(0)
        _check(lib.tilemix_paged_decode_workspace_size(c, heads, ctypes.byref(n)))
        nbytes = n.value
        if nbytes:
            workspace = _alloc_like(stream, Q, (nbytes,), torch.uint8)
    else:
        if not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the pool's device")
        nbytes = workspace.numel() * workspace.element_size()
    _check_call(lib.tilemix_paged_decode(
        c, fmt, heads, scale if scale is not None else 1.0 / math.sqrt(d), window, Q.data_ptr(), q_stride, O.data_ptr(),
        _ptr(lse), _ptr(workspace), nbytes, handle))
    return (O, lse) if return_lse else O


class PageList(NamedTuple):
    """The free pages of a pool for ``tilemix_paged_reserve``: ids int32 CUDA [capacity], a ring, and state int32 CUDA [4]:
    where the first free page lies, how many there are, the sequences that the last call refused, 0."""
    ids: object
    state: object

    @staticmethod
    def full(pages: int, device="cuda") -> "PageList":
        """All pages of a pool of ``pages`` are free."""
        import torch
        return PageList(torch.arange(pages, dtype=torch.int32, device=device),
                        torch.tensor([0, pages, 0, 0], dtype=torch.int32, device=device))


class Reserved(NamedTuple):
    """What tilemix_paged_reserve returns: the new lengths int32 [B], prefix sums of the new tokens int32 [B + 1], and with
    ``total`` the position (int32) and slot (int64) of each."""
    seqlens: object
    cu_seqlens: object
    positions: object
    slots: object


def tilemix_paged_reserve(pages: PageList, page_table, seqlens, wanted, page_size: int, *, window: int = 0,
                          first_held=None, total: int | None = None, state_out=None, seqlens_out=None, cu_seqlens=None, positions=None,
                          slots=None, stream=None) -> Reserved:
    """Move pages between ``page_table`` (int32 CUDA [B, max_pages]) and the free ``pages`` so that sequences of
    ``seqlens`` tokens (int32 CUDA [B]) have room for ``wanted`` (int32 CUDA [B]; 0: done).  A sequence whose pages are
    not there keeps its length.  ``seqlens`` and the list's state are updated in place, unless ``seqlens_out`` (int32
    [B]) or ``state_out`` (int32 [4]) is given.  With ``total`` rows the new tokens' positions and slots
    (page * page_size + slot) are written, -1 behind the last one; tensors for the results are allocated when not
    given.  ``window``: a sliding window of that many tokens, whose pages go back when it has left them; ``first_held``
    (int32 [B], 0 at the start) then keeps the first page-table entry that each sequence still holds.  Readers of a page
    are not counted: tables whose sequences share pages are not for this call.  Results may overlap no other tensor of the call,
    but seqlens_out may be ``seqlens`` or ``wanted`` and state_out the list's state."""
    torch = _torch()
    ids, state = pages
    if not isinstance(ids, torch.Tensor) or not ids.is_cuda:
        raise TypeError("the list's ids must be a CUDA (HIP) tensor")
    dev, i32 = ids.get_device(), torch.int32
    if ids.ndim != 1:
        raise ValueError("the list's ids must be [capacity]")
    _require_dense(ids, i32, ids.shape, dev, "the list's ids")
    _require_dense(state, i32, (4,), dev, "the list's state")
    if getattr(page_table, "ndim", None) != 2:
        raise ValueError("page_table must be a tensor [B, max_pages]")
    shape = page_table.shape
    _require_like(page_table, i32, shape, dev, "page_table")
    B = shape[0]
    _require_dense(seqlens, i32, (B,), dev, "seqlens")
    _require_dense(wanted, i32, (B,), dev, "wanted")
    if (first_held is None) != (window == 0):
        raise ValueError("first_held goes with a window, and with it only")
    if first_held is not None:
        _require_dense(first_held, i32, (B,), dev, "first_held")
    if total is None and (positions is not None or slots is not None):
        raise ValueError("total is needed with positions or slots")
    _int32(page_size, "page_size"), _int32(window, "window"), _int32(total or 0, "total")
    other = _elsewhere(dev)
    if other is not None:
        with other:
            return tilemix_paged_reserve(pages, page_table, seqlens, wanted, page_size, window=window, first_held=first_held,
                                         total=total, state_out=state_out,
                                         seqlens_out=seqlens_out, cu_seqlens=cu_seqlens, positions=positions, slots=slots, stream=stream)
    handle = _stream_on(stream, dev)
    if state_out is None:
        state_out = state
    else:
        _require_dense(state_out, i32, (4,), dev, "state_out")
    if seqlens_out is None:
        seqlens_out = seqlens
    else:
        _require_dense(seqlens_out, i32, (B,), dev, "seqlens_out")
    if cu_seqlens is None:
        cu_seqlens = _alloc_like(stream, ids, (B + 1,))
    else:
        _require_dense(cu_seqlens, i32, (B + 1,), dev, "cu_seqlens")
    if total is not None:
        if total < 0:
            raise ValueError("total must be >= 0")
        if positions is None:
            positions = _alloc_like(stream, ids, (total,))
        else:
            _require_dense(positions, i32, (total,), dev, "positions")
        if slots is None:
            slots = _alloc_like(stream, ids, (total,), torch.int64)
        else:
            _require_dense(slots, torch.int64, (total,), dev, "slots")
    _check(load_library().tilemix_paged_reserve(
        page_size, B, shape[1], page_table.data_ptr(),
        shape[1] if page_table.is_contiguous() else _outer_stride(shape, page_table.stride(), 1, "page_table"), seqlens.data_ptr(),
        wanted.data_ptr(), window, _ptr(first_held), ids.data_ptr(), ids.shape[0], state.data_ptr(), state_out.data_ptr(), seqlens_out.data_ptr(),
        cu_seqlens.data_ptr(), _ptr(positions), _ptr(slots), total or 0, handle))
    return Reserved(seqlens_out, cu_seqlens, positions, slots)


# ------------------------------------------------------------------------- rotary positions

_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}
_ROTARY = struct.Struct("<7ifQ")            # tilemix_rotary_params
_ROTARY_SCALING = struct.Struct("<2i4di4x")  # tilemix_rotary_scaling


def tilemix_rotary_frequencies(rotary_dim: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                               original_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(inv_freq float64 [rotary_dim / 2] on ``device``, magnitude) for tilemix_rotary.  ``scaling`` for contexts that are
    ``factor`` times as long as those trained on: "linear" (positions / factor), "ntk" (a larger base) or "yarn" (arXiv
    2309.00071, with ``original_len`` tokens trained on: frequencies of more than ``beta_fast`` rotations over them are
    kept, those of fewer than ``beta_slow`` divided, and those in between mixed by their rotations, as in the paper; a model
    whose training mixed them by the pair's number needs its own inv_freq)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {list(_SCALINGS)}, got {scaling!r}")
    import torch
    c = _ROTARY_SCALING.pack(_SCALINGS[scaling], _int32(rotary_dim, "rotary_dim"), base, factor, beta_fast, beta_slow,
                             _int32(original_len, "original_len"))
    out = (ctypes.c_double * 64)()
    magnitude = ctypes.c_float()
    _check(load_library().tilemix_rotary_frequencies(c, out, ctypes.byref(magnitude)))
    return torch.tensor(out[:rotary_dim // 2], dtype=torch.float64, device=device), magnitude.value


def tilemix_rotary(Q, K, inv_freq, positions=None, *, seqlens_k=None, cu_seqlens=None, layout: str = "half",
                   magnitude: float = 1.0, inverse: bool = False, Q_out=None, K_out=None, stream=None):
    """Rotary positions on Q and K, float16 or bfloat16 CUDA [total, H, d] or [B, L, H, d] (K may be None; tokens may
    lie any multiple of 8 elements apart).  inv_freq: float64 CUDA [rotary_dim / 2], of tilemix_rotary_frequencies; channels from
    rotary_dim on stay as they are.  Rows have the ``positions`` int32 CUDA [total] or [B, L], or are the last ones of
    sequences of ``seqlens_k`` tokens (int32 CUDA [B]), packed by ``cu_seqlens`` (int32 CUDA [B + 1]) or L of each, as in
    tilemix_paged_append.  Pairs are channels i and i + rotary_dim / 2 (layout "half") or 2 i and 2 i + 1
    ("interleaved").  Returns (Q_out, K_out), allocated when not given; they may be Q and K.  Rows with a negative
    position, or that no sequence owns, are not written.  ``inverse``: turned the other way, which makes gradients of Q and
    K out of those of the results (which carry none themselves: nothing here is recorded for autograd)."""
    torch = _torch()
    if not isinstance(Q, torch.Tensor) or not Q.is_cuda:
        raise TypeError("Q must be a CUDA (HIP) tensor")
    dtype, shape, dev = Q.dtype, Q.shape, Q.get_device()
    fmt = _format(dtype)
    if fmt not in (0, 1):
        raise TypeError(f"Q must be float16 or bfloat16, got {dtype}")
    if len(shape) not in (3, 4):
        raise ValueError("Q and K must be [total, H, d] or [B, L, H, d]")
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {list(_LAYOUTS)}, got {layout!r}")
    rows, (Hq, d) = shape[:-2], shape[-2:]
    Hk, k_shape = 0, None
    if K is None:
        if K_out is not None:
            raise ValueError("K_out is given without K")
    else:
        if getattr(K, "ndim", None) != len(shape):
            raise ValueError("K must have as many dimensions as Q")
        Hk = K.shape[-2]
        k_shape = (*rows, Hk, d)
        _require_like(K, dtype, k_shape, dev, "K")
    if getattr(inv_freq, "ndim", None) != 1:
        raise ValueError("inv_freq must be a tensor [rotary_dim / 2]")
    _require_dense(inv_freq, torch.float64, inv_freq.shape, dev, "inv_freq")
    total = rows[0] if len(rows) == 1 else rows[0] * rows[1]
    batch, pos, lens, cu = 1, None, None, None
    if positions is not None:
        if seqlens_k is not None or cu_seqlens is not None:
            raise ValueError("positions and seqlens_k exclude each other")
        _require_dense(positions, torch.int32, rows, dev, "positions")
        pos = positions.data_ptr()
    else:
        if seqlens_k is None:
            raise ValueError("positions or seqlens_k is needed")
        batch = rows[0] if len(rows) == 2 else getattr(seqlens_k, "shape", (0,))[0]
        _require_dense(seqlens_k, torch.int32, (batch,), dev, "seqlens_k")
        lens = seqlens_k.data_ptr()
        if (cu_seqlens is None) == (len(rows) == 1):
            raise ValueError("cu_seqlens goes with [total, H, d], and with it only")
        if cu_seqlens is not None:
            _require_dense(cu_seqlens, torch.int32, (batch + 1,), dev, "cu_seqlens")
            cu = cu_seqlens.data_ptr()
    _int32(total, "total")
    other = _elsewhere(dev)
    if other is not None:
        with other:
            return tilemix_rotary(Q, K, inv_freq, positions, seqlens_k=seqlens_k, cu_seqlens=cu_seqlens, layout=layout,
                                  magnitude=magnitude, inverse=inverse, Q_out=Q_out, K_out=K_out, stream=stream)
    handle = _stream_on(stream, dev)
    if Q_out is None:
        Q_out = _alloc_like(stream, Q, shape)
    else:
        _require_like(Q_out, dtype, shape, dev, "Q_out")
    k = ko = None
    ks = kos = 0
    if K is not None:
        if K_out is None:
            K_out = _alloc_like(stream, K, k_shape)
        else:
            _require_like(K_out, dtype, k_shape, dev, "K_out")
        k, ks, ko, kos = K.data_ptr(), _row_stride(K, k_shape, "K"), K_out.data_ptr(), _row_stride(K_out, k_shape, "K_out")
    c = _ROTARY.pack(fmt, _LAYOUTS[layout], d, 2 * inv_freq.shape[0], Hq, Hk, 1 if inverse else 0, magnitude, inv_freq.data_ptr())
    _check(load_library().tilemix_rotary(c, pos, lens, cu, batch, total, Q.data_ptr(), _row_stride(Q, shape, "Q"), Q_out.data_ptr(),
                                         _row_stride(Q_out, shape, "Q_out"), k, ks, ko, kos, handle))
    return Q_out, K_out
