"""Python binding of libsdq, the GB300 Sigma-Delta-quantized linear layer.

Thin ctypes layer over the C ABI in ``include/sdq.h``: the functions below
carry the C names and only marshal arguments (pointers, sizes, streams).  All
compute runs in the CUDA kernels of ``libsdq.so``; there is no CPU path.  If
the library is missing, every call raises ``RuntimeError`` -- build it with
``python -m paper_2510_03275_gb300.build``.

Tensors are PyTorch tensors (device memory and streams only).  bf16
activations are passed as ``torch.bfloat16`` tensors; codes as ``torch.int32``
tensors holding the uint32 words.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from fractions import Fraction
from typing import NamedTuple

__all__ = [
    "SDQ_OK", "SDQ_BINARY", "SDQ_TERNARY", "SDQ_ALPHA_MAXABS", "SDQ_ALPHA_MEANABS",
    "SdqError", "LayerDesc", "lib", "library_path",
    "sdq_plan_create", "sdq_plan_destroy", "sdq_k_eff", "sdq_plain_bytes", "sdq_tiled_bytes",
    "sdq_workspace_bytes", "sdq_build_tables", "sdq_build_gptq_table", "sdq_decode_launch_shape", "sdq_encode_rows", "sdq_gptq_workspace_bytes",
    "sdq_encode_rows_gptq", "sdq_base3_bytes", "sdq_pack_base3", "sdq_unpack_base3", "sdq_pack", "sdq_unpack",
    "sdq_prep_activations", "sdq_contract", "sdq_contract_add", "sdq_linear_forward", "sdq_read_prep",
    "sdq_workspace_status", "sdq_linear_forward_noalloc", "sdq_noalloc_scratch_bytes", "sdq_noalloc_status",
    "sdq_forward_kernels", "sdq_forward_route", "sdq_status_string", "Plan",
    "SDQ_F32", "SDQ_BF16", "CacheDesc", "Batch", "Rope", "KVCache",
    "sdq_cache_bytes", "sdq_cache_create", "sdq_cache_destroy", "sdq_rope_table", "sdq_cache_append",
    "sdq_attention_workspace_bytes", "sdq_attention", "sdq_attention_status",
    "sdq_sample", "sample",
    "HeadNorm", "sdq_cache_append_norm", "PagePool", "PageStep", "sdq_pages_step", "sdq_adjust_logits", "adjust_logits",
    "sdq_attention_window", "sdq_attention_window_workspace_bytes",
]

SDQ_OK = 0
SDQ_BINARY = 1
SDQ_TERNARY = 2
SDQ_ALPHA_MAXABS = 0
SDQ_ALPHA_MEANABS = 1
SDQ_F32 = 0
SDQ_BF16 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libsdq.so")


class SdqError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = lib().sdq_status_string(status).decode() if _lib is not None else str(status)
        super().__init__(f"{where}: {msg}")
        self.status = status


class _Desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_out", "k_in", "block", "osr_num", "osr_den", "quantizer", "hadamard",
                 "alpha_mode")]


@dataclass(frozen=True)
class LayerDesc:
    """Mirror of ``sdq_layer_desc``: OSR is a Fraction (num/den)."""
    n_out: int
    k_in: int
    block: int
    osr: Fraction
    quantizer: int = SDQ_TERNARY
    hadamard: int = 1
    alpha_mode: int = SDQ_ALPHA_MAXABS

    def c(self) -> _Desc:
        o = Fraction(self.osr)
        return _Desc(self.n_out, self.k_in, self.block, o.numerator, o.denominator,
                     self.quantizer, self.hadamard, self.alpha_mode)

    @property
    def n_b(self) -> int:
        return int(self.block * Fraction(self.osr))


class _CacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("kv_heads", "head_dim", "page_tokens", "n_pages")]


class _Batch(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("n_seqs", "n_tokens", "max_new", "max_own", "page_stride", "prefix_len")]
                + [(n, ctypes.c_void_p) for n in ("token_start", "own_len", "pages", "prefix_pages")])


class _Rope(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("n_pos", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


class _HeadNorm(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("q_per_head", ctypes.c_int32), ("k_per_head", ctypes.c_int32),
                ("eps", ctypes.c_float)]


# (packed by `struct`: a third of the time of a ctypes structure)
_ADJUST = struct.Struct("10P4q3i4x")   # sdq_adjust
_PAGES = struct.Struct("7i11P")        # sdq_pages


@dataclass(frozen=True)
class CacheDesc:
    """Mirror of ``sdq_cache_desc``."""
    kv_heads: int
    head_dim: int
    page_tokens: int
    n_pages: int

    def c(self) -> _CacheDesc:
        return _CacheDesc(self.kv_heads, self.head_dim, self.page_tokens, self.n_pages)

    @property
    def shape(self):
        """Of each of the two arrays: (page, key head, token of the page, element)."""
        return self.n_pages, self.kv_heads, self.page_tokens, self.head_dim


_lib = None
_vp, _sz, _i32, _i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
_SIGS = {
    "sdq_plan_create": (ctypes.c_int, [ctypes.POINTER(_Desc), _vp, ctypes.POINTER(_vp)]),
    "sdq_plan_destroy": (ctypes.c_int, [_vp]),
    "sdq_k_eff": (_i64, [ctypes.POINTER(_Desc)]),
    "sdq_plain_bytes": (_sz, [ctypes.POINTER(_Desc)]),
    "sdq_tiled_bytes": (_sz, [ctypes.POINTER(_Desc)]),
    "sdq_workspace_bytes": (_sz, [_vp, _i32]),
    "sdq_build_tables": (ctypes.c_int, [ctypes.POINTER(_Desc), _vp, _vp, _vp]),
    "sdq_build_gptq_table": (ctypes.c_int, [ctypes.POINTER(_Desc), _vp, _vp]),
    "sdq_decode_launch_shape": (ctypes.c_int, [ctypes.POINTER(_Desc), _i32, _i32, _vp]),
    "sdq_encode_rows": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "sdq_gptq_workspace_bytes": (ctypes.c_size_t, [_vp]),
    "sdq_base3_bytes": (ctypes.c_size_t, [ctypes.POINTER(_Desc)]),
    "sdq_pack_base3": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "sdq_unpack_base3": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "sdq_encode_rows_gptq": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "sdq_pack": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "sdq_unpack": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "sdq_prep_activations": (ctypes.c_int, [_vp, _vp, _i32, _vp, _sz, _vp]),
    "sdq_contract": (ctypes.c_int, [_vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "sdq_contract_add": (ctypes.c_int, [_vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "sdq_linear_forward": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "sdq_read_prep": (ctypes.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "sdq_workspace_status": (ctypes.c_int, [_vp, _i32, _vp, _vp]),
    "sdq_forward_kernels": (ctypes.c_int, [_vp, _i32, _vp]),
    "sdq_forward_route": (ctypes.c_int, [_vp, _i32]),
    "sdq_linear_forward_noalloc": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i32, _vp, _vp]),
    "sdq_noalloc_status": (ctypes.c_int, [_vp, _i32, _vp]),
    "sdq_noalloc_scratch_bytes": (_sz, []),
    "sdq_cache_bytes": (_sz, [ctypes.POINTER(_CacheDesc)]),
    "sdq_cache_create": (ctypes.c_int, [ctypes.POINTER(_CacheDesc), _vp, _vp, ctypes.POINTER(_vp)]),
    "sdq_cache_destroy": (ctypes.c_int, [_vp]),
    "sdq_rope_table": (ctypes.c_int, [_i32, _i32, ctypes.c_double, _vp, _vp]),
    "sdq_cache_append": (ctypes.c_int, [_vp, _vp, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _vp, _vp]),
    "sdq_cache_append_norm": (ctypes.c_int, [_vp, _vp, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _vp, _vp, _vp]),
    "sdq_attention_workspace_bytes": (_sz, [_vp, _vp, _i32]),
    "sdq_attention": (ctypes.c_int, [_vp, _vp, _i32, _vp, _i64, ctypes.c_float, _vp, _vp, _vp, _sz, _vp]),
    "sdq_attention_window_workspace_bytes": (_sz, [_vp, _vp, _i32, _i32, _i32]),
    "sdq_attention_window": (ctypes.c_int, [_vp, _vp, _i32, _vp, _i64, ctypes.c_float, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "sdq_attention_status": (ctypes.c_int, [_vp, _vp]),
    "sdq_sample": (ctypes.c_int, [_vp, _i32, _i32, _i32, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sdq_pages_step": (ctypes.c_int, [_vp, _vp]),
    "sdq_adjust_logits": (ctypes.c_int, [_vp, _i32, _i32, _i32, _i64, _vp, _vp, _i64, _vp]),
    "sdq_status_string": (ctypes.c_char_p, [ctypes.c_int]),
}


def lib():
    """Load libsdq.so (once); raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(library_path):
            raise RuntimeError(f"libsdq.so not found at {library_path}; run "
                               "`python -m paper_2510_03275_gb300.build` (CUDA toolkit needed)")
        L = ctypes.CDLL(library_path)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(st: int, where: str):
    if st != SDQ_OK:
        raise SdqError(st, where)


# Pointers and streams go to the C functions as plain ints (their argument
# types convert them).  A decode call is a few microseconds of launches, so
# its marshalling counts: with ctypes objects per pointer and a torch.cuda.Stream
# per call, Plan.forward spent 12.8 of its 16.7 us of host time there.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _first_current_stream() -> int:
    """The handle of the current device's current stream; from the second call
    on straight from the binding torch keeps for generated code, where this
    torch has it."""
    global _current_stream
    import torch
    handle = torch.cuda.current_stream().cuda_stream   # (initializes CUDA)
    raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and dev is not None and raw(dev()) == handle:
        _current_stream = lambda: raw(dev())
    else:
        _current_stream = lambda: torch.cuda.current_stream().cuda_stream
    return handle


_current_stream = _first_current_stream


def _stream(stream):
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype, device, stream):
    """Device memory that belongs to the stream a call runs on (a block that the current stream still uses is not
    handed out to another)."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(getattr(stream, "cuda_stream", stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _first_current_device() -> int:
    """The current device; once CUDA is initialized straight from the binding that torch's own call ends in, where this
    torch has it."""
    global _current_device
    import torch
    device, raw = torch.cuda.current_device(), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and torch.cuda.is_initialized() and raw() == device:
        _current_device = raw
    return device


_current_device = _first_current_device


def _check_devices(where, first, *others):
    """Raise unless the tensors (None: left out) are all on the current device, on which the kernels run."""
    device = first.get_device()
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError(f"{where}: tensors on different devices")
    if device != _current_device():
        raise ValueError(f"{where}: the tensors are not on the current device")


# ------------------------------------------------------------- C-ABI names
def sdq_plan_create(desc: LayerDesc, had_signs=None) -> int:
    import numpy as np
    d = desc.c()
    h = ctypes.c_void_p()
    signs = None
    if had_signs is not None:
        signs = np.ascontiguousarray(had_signs, dtype=np.int8)
    st = lib().sdq_plan_create(ctypes.byref(d),
                               None if signs is None else signs.ctypes.data_as(_vp),
                               ctypes.byref(h))
    _check(st, "sdq_plan_create")
    return h.value


def sdq_plan_destroy(plan: int):
    _check(lib().sdq_plan_destroy(plan), "sdq_plan_destroy")


def sdq_k_eff(desc: LayerDesc) -> int:
    return lib().sdq_k_eff(ctypes.byref(desc.c()))


def sdq_plain_bytes(desc: LayerDesc) -> int:
    return lib().sdq_plain_bytes(ctypes.byref(desc.c()))


def sdq_tiled_bytes(desc: LayerDesc) -> int:
    return lib().sdq_tiled_bytes(ctypes.byref(desc.c()))


def sdq_workspace_bytes(plan: int, M: int) -> int:
    return lib().sdq_workspace_bytes(plan, M)


def sdq_build_tables(desc: LayerDesc, had_signs=None):
    """Host-only: (A_enc, G) as float32 numpy arrays (n_b x B)."""
    import numpy as np
    a = np.zeros((desc.n_b, desc.block), np.float32)
    g = np.zeros((desc.n_b, desc.block), np.float32)
    signs = None if had_signs is None else np.ascontiguousarray(had_signs, dtype=np.int8)
    st = lib().sdq_build_tables(ctypes.byref(desc.c()),
                                None if signs is None else signs.ctypes.data_as(_vp),
                                a.ctypes.data_as(_vp), g.ctypes.data_as(_vp))
    _check(st, "sdq_build_tables")
    return a, g


def sdq_build_gptq_table(desc: LayerDesc, had_signs=None):
    """Host-only: the fp32 G of the GPTQ block reconstruction (n_b x B)."""
    import numpy as np
    g = np.zeros((desc.n_b, desc.block), np.float32)
    signs = None if had_signs is None else np.ascontiguousarray(had_signs, dtype=np.int8)
    st = lib().sdq_build_gptq_table(ctypes.byref(desc.c()), None if signs is None else signs.ctypes.data_as(_vp),
                                    g.ctypes.data_as(_vp))
    _check(st, "sdq_build_gptq_table")
    return g


_SHAPE_KEYS = ("T", "NP", "S", "P", "CB", "ring", "sb", "nbuf", "smem", "slot_bytes", "b_bytes", "ss",
               "smem_limit", "npipe", "ns", "bstream")


def sdq_decode_launch_shape(desc: LayerDesc, M: int, sm_count: int) -> dict:
    """Host-only: the decode launch shape at batch M (include/sdq.h)."""
    import numpy as np
    out = np.zeros(len(_SHAPE_KEYS), np.int64)
    _check(lib().sdq_decode_launch_shape(ctypes.byref(desc.c()), M, sm_count, out.ctypes.data_as(_vp)),
           "sdq_decode_launch_shape")
    return dict(zip(_SHAPE_KEYS, (int(v) for v in out)))


def sdq_encode_rows(plan, W, codes_plain, alpha, stream=None):
    _check(lib().sdq_encode_rows(plan, _ptr(W), _ptr(codes_plain), _ptr(alpha), _stream(stream)),
           "sdq_encode_rows")


def sdq_gptq_workspace_bytes(plan) -> int:
    return int(lib().sdq_gptq_workspace_bytes(plan))


def sdq_encode_rows_gptq(plan, W, U, codes_plain, alpha, ws, stream=None):
    _check(lib().sdq_encode_rows_gptq(plan, _ptr(W), _ptr(U), _ptr(codes_plain), _ptr(alpha), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)),
           "sdq_encode_rows_gptq")


def sdq_base3_bytes(desc: LayerDesc) -> int:
    return int(lib().sdq_base3_bytes(ctypes.byref(desc.c())))


def sdq_pack_base3(plan, codes_plain, codes_base3, stream=None):
    _check(lib().sdq_pack_base3(plan, _ptr(codes_plain), _ptr(codes_base3), _stream(stream)), "sdq_pack_base3")


def sdq_unpack_base3(plan, codes_base3, codes_plain, bad_count=None, stream=None):
    _check(lib().sdq_unpack_base3(plan, _ptr(codes_base3), _ptr(codes_plain),
                                  None if bad_count is None else _ptr(bad_count), _stream(stream)),
           "sdq_unpack_base3")


def sdq_pack(plan, codes_plain, codes_tiled, stream=None):
    _check(lib().sdq_pack(plan, _ptr(codes_plain), _ptr(codes_tiled), _stream(stream)), "sdq_pack")


def sdq_unpack(plan, codes_tiled, codes_plain, bad_count=None, stream=None):
    _check(lib().sdq_unpack(plan, _ptr(codes_tiled), _ptr(codes_plain), _ptr(bad_count),
                            _stream(stream)), "sdq_unpack")


def sdq_prep_activations(plan, x, M, ws, stream=None):
    _check(lib().sdq_prep_activations(plan, _ptr(x), M, _ptr(ws), ws.numel() * ws.element_size(),
                                      _stream(stream)), "sdq_prep_activations")


def sdq_contract(plan, codes_tiled, alpha, M, y, ws, stream=None):
    _check(lib().sdq_contract(plan, _ptr(codes_tiled), _ptr(alpha), M, _ptr(y), _ptr(ws),
                              ws.numel() * ws.element_size(), _stream(stream)), "sdq_contract")


def sdq_contract_add(plan, codes_tiled, alpha, M, y, ws, stream=None):
    """y += the contraction (M <= 64; float reductions, order not fixed)."""
    _check(lib().sdq_contract_add(plan, _ptr(codes_tiled), _ptr(alpha), M, _ptr(y), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(stream)), "sdq_contract_add")


def sdq_linear_forward(plan, codes_tiled, alpha, x, M, y, ws, stream=None):
    _check(lib().sdq_linear_forward(plan, _ptr(codes_tiled), _ptr(alpha), _ptr(x), M, _ptr(y),
                                    _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "sdq_linear_forward")


def sdq_read_prep(plan, M, ws, out, stream=None):
    _check(lib().sdq_read_prep(plan, M, _ptr(ws), _ptr(out), _stream(stream)), "sdq_read_prep")


def sdq_workspace_status(plan, M, ws, stream=None) -> int:
    """Synchronize and return the status of the last decode using ``ws``."""
    return lib().sdq_workspace_status(plan, M, _ptr(ws), _stream(stream))


def sdq_forward_kernels(plan, M, x) -> int:
    """Number of kernels sdq_linear_forward launches (2)."""
    return lib().sdq_forward_kernels(plan, M, _ptr(x))


def sdq_forward_route(plan, M) -> int:
    """Route of sdq_linear_forward at batch M: 1 decode, 2 code-domain
    prefill, 3 dense (weights rebuilt, then one GEMM); see include/sdq.h."""
    return lib().sdq_forward_route(plan, M)


def sdq_linear_forward_noalloc(plan, codes_tiled, alpha, x, M, y, stream=None):
    """Decode forward (M <= 64) using the library's own device scratch array
    instead of a caller workspace; see include/sdq.h for its rules."""
    _check(lib().sdq_linear_forward_noalloc(plan, _ptr(codes_tiled), _ptr(alpha), _ptr(x), M,
                                            _ptr(y), _stream(stream)),
           "sdq_linear_forward_noalloc")


def sdq_noalloc_scratch_bytes() -> int:
    return lib().sdq_noalloc_scratch_bytes()


def sdq_noalloc_status(plan, M, stream=None) -> int:
    """Synchronize and return the status of the last allocation-free call
    with this plan and M on the current device (SDQ_OK or a negative status)."""
    return lib().sdq_noalloc_status(plan, M, _stream(stream))


def sdq_cache_bytes(desc: CacheDesc) -> int:
    return lib().sdq_cache_bytes(ctypes.byref(desc.c()))


def sdq_cache_create(desc: CacheDesc, k_pages, v_pages) -> int:
    h = ctypes.c_void_p()
    _check(lib().sdq_cache_create(ctypes.byref(desc.c()), _ptr(k_pages), _ptr(v_pages), ctypes.byref(h)),
           "sdq_cache_create")
    return h.value


def sdq_cache_destroy(cache: int):
    _check(lib().sdq_cache_destroy(cache), "sdq_cache_destroy")


def sdq_rope_table(n_pos: int, dim: int, base: float = 10000.0):
    """Host-only: (cos, sin) as float32 numpy arrays (n_pos x dim / 2)."""
    import numpy as np
    cos, sin = (np.zeros((max(n_pos, 0), max(dim, 0) // 2), np.float32) for _ in range(2))
    _check(lib().sdq_rope_table(n_pos, dim, base, cos.ctypes.data_as(_vp), sin.ctypes.data_as(_vp)), "sdq_rope_table")
    return cos, sin


def _dtype(t) -> int:
    """The ``sdq_dtype`` of a tensor; -1 (which every entry point refuses) for other types."""
    import torch
    return SDQ_F32 if t.dtype == torch.float32 else SDQ_BF16 if t.dtype == torch.bfloat16 else -1


def sdq_cache_append(cache, batch, q_heads, q, k, v, rope, q_out, stream=None):
    """q, k, v: one row per token, of one type; their row strides are the tensors'."""
    _check(lib().sdq_cache_append(cache, batch.ref, q_heads, *_rows_of(q, k, v), rope.ref, q_out.data_ptr(), _stream(stream)),
           "sdq_cache_append")


def _rows_of(q, k, v):
    kind = _dtype(q) if k.dtype == v.dtype == q.dtype else -1
    # (a single row has no stride of its own)
    ldq, ldk, ldv = (q.shape[1], k.shape[1], v.shape[1]) if q.shape[0] == 1 else (q.stride()[0], k.stride()[0], v.stride()[0])
    return q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, kind


def sdq_cache_append_norm(cache, batch, q_heads, q, k, v, rope, norm, q_out, stream=None):
    """As sdq_cache_append, the heads of q and k normalised by `norm` (a HeadNorm)."""
    _check(lib().sdq_cache_append_norm(cache, batch.ref, q_heads, *_rows_of(q, k, v), rope.ref, norm.ref, q_out.data_ptr(),
                                       _stream(stream)), "sdq_cache_append_norm")


def sdq_attention_workspace_bytes(cache, batch, q_heads) -> int:
    return lib().sdq_attention_workspace_bytes(cache, batch.ref, q_heads)


def sdq_attention(cache, batch, q_heads, q, ldq, scale, out, lse, ws, stream=None):
    _check(lib().sdq_attention(cache, batch.ref, q_heads, q.data_ptr(), ldq, scale, out.data_ptr(), _ptr(lse),
                               ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)), "sdq_attention")


def sdq_attention_window_workspace_bytes(cache, batch, q_heads, window, sinks) -> int:
    return lib().sdq_attention_window_workspace_bytes(cache, batch.ref, q_heads, window, sinks)


def sdq_attention_window(cache, batch, q_heads, q, ldq, scale, window, sinks, out, lse, ws, stream=None):
    _check(lib().sdq_attention_window(cache, batch.ref, q_heads, q.data_ptr(), ldq, scale, window, sinks, out.data_ptr(),
                                      _ptr(lse), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)),
           "sdq_attention_window")


def sdq_attention_status(ws, stream=None) -> int:
    """Synchronize and return the status of the last attention call on ``ws``."""
    return lib().sdq_attention_status(_ptr(ws), _stream(stream))


def sdq_sample(logits, u, temperature, top_k, top_p, min_p, tokens, stream=None):
    """logits: rows x vocab, adjacent in a row; any of the four settings may be None."""
    rows, vocab = logits.shape
    _check(lib().sdq_sample(logits.data_ptr(), _dtype(logits), rows, vocab, logits.stride(0) if rows > 1 else vocab,
                            u.data_ptr(), _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), tokens.data_ptr(),
                            _stream(stream)), "sdq_sample")


def sdq_pages_step(step: bytes, stream=None):
    """step: the bytes of an ``sdq_pages``."""
    _check(lib().sdq_pages_step(step, _stream(stream)), "sdq_pages_step")


def sdq_adjust_logits(logits, adjust: bytes, out, stream=None):
    """logits, out: rows x vocab of one type, adjacent in a row; adjust: the bytes of an ``sdq_adjust``."""
    rows, vocab = logits.shape
    _check(lib().sdq_adjust_logits(logits.data_ptr(), _dtype(logits), rows, vocab, logits.stride()[0] if rows > 1 else vocab,
                                   adjust, out.data_ptr(), out.stride()[0] if rows > 1 else vocab, _stream(stream)),
           "sdq_adjust_logits")


def sdq_status_string(status: int) -> str:
    return lib().sdq_status_string(status).decode()


# ------------------------------------------------------------ convenience
class Plan:
    """Owns an ``sdq_plan`` plus the device buffers of one quantized layer."""

    def __init__(self, desc: LayerDesc, had_signs=None):
        self.desc = desc
        self.handle = sdq_plan_create(desc, had_signs)
        self.k_eff = sdq_k_eff(desc)

    def close(self):
        if self.handle:
            sdq_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc_plain(self, device="cuda"):
        import torch
        return torch.empty(sdq_plain_bytes(self.desc) // 4, dtype=torch.int32, device=device)

    def alloc_tiled(self, device="cuda"):
        import torch
        return torch.empty(sdq_tiled_bytes(self.desc) // 4, dtype=torch.int32, device=device)

    def alloc_workspace(self, M, device="cuda"):
        import torch
        return torch.empty(sdq_workspace_bytes(self.handle, M), dtype=torch.uint8, device=device)

    def encode(self, W, stream=None):
        """W (n_out x k_in fp32, device) -> (plain codes, alpha)."""
        import torch
        codes = self.alloc_plain(W.device)
        alpha = torch.empty(self.desc.n_out, dtype=torch.float32, device=W.device)
        sdq_encode_rows(self.handle, W.contiguous(), codes, alpha, stream)
        return codes, alpha

    def encode_gptq(self, W, U, stream=None):
        """W (n_out x k_in fp32, device), U (k_in x k_in fp32, device, upper,
        U^T U = H^-1) -> (plain codes, alpha) with GPTQ block compensation."""
        import torch
        codes = self.alloc_plain(W.device)
        alpha = torch.empty(self.desc.n_out, dtype=torch.float32, device=W.device)
        ws = torch.empty(sdq_gptq_workspace_bytes(self.handle), dtype=torch.uint8, device=W.device)
        sdq_encode_rows_gptq(self.handle, W.contiguous(), U.contiguous(), codes, alpha, ws, stream)
        return codes, alpha

    def pack(self, plain, stream=None):
        tiled = self.alloc_tiled(plain.device)
        sdq_pack(self.handle, plain, tiled, stream)
        return tiled

    def forward(self, tiled, alpha, x, ws=None, stream=None):
        """x (M x k_in bf16, device) -> y (M x n_out fp32)."""
        import torch
        M = x.shape[0]
        if ws is None:
            ws = self.alloc_workspace(M, x.device)
        y = torch.empty((M, self.desc.n_out), dtype=torch.float32, device=x.device)
        sdq_linear_forward(self.handle, tiled, alpha, x.contiguous(), M, y, ws, stream)
        return y


class Batch:
    """Mirror of ``sdq_batch``: one step's tokens, the pages of their sequences
    and the prefix that all of them share.  Holds the four int32 tensors."""

    def __init__(self, token_start, own_len, pages, n_tokens, max_new, max_own, prefix_pages=None, prefix_len=0):
        import torch
        for name, t, dims in (("token_start", token_start, 1), ("own_len", own_len, 1), ("pages", pages, 2),
                              ("prefix_pages", prefix_pages, 1)):
            if t is not None and (t.dtype != torch.int32 or t.dim() != dims or not t.is_cuda
                                  or (t.numel() > 0 and t.stride(-1) != 1)):
                raise ValueError(f"Batch: {name} must be a {dims}-d int32 CUDA tensor with adjacent elements")
        n_seqs = own_len.shape[0]
        if token_start.shape[0] != n_seqs + 1 or pages.shape[0] != n_seqs:
            raise ValueError("Batch: token_start needs one entry more than own_len, pages one row for each")
        self.n_seqs, self.n_tokens, self.max_new, self.max_own = n_seqs, n_tokens, max_new, max_own
        self.prefix_len = prefix_len
        self.tensors = (token_start, own_len, pages, prefix_pages)
        self.device_index = own_len.get_device()
        if any(t is not None and t.get_device() != self.device_index for t in self.tensors):
            raise ValueError("Batch: tensors on different devices")
        self.page_columns = pages.shape[1]
        self._c = _Batch(n_seqs, n_tokens, max_new, max_own, pages.stride(0) if n_seqs > 1 else pages.shape[1], prefix_len,
                         token_start.data_ptr(), own_len.data_ptr(), pages.data_ptr() or None,
                         None if prefix_pages is None else prefix_pages.data_ptr() or None)
        self.ref = ctypes.addressof(self._c)
        self._checked = None

    def check(self, page_tokens: int):
        """Raise where the page tables are too short for max_own or prefix_len."""
        if self._checked == page_tokens:   # (neither changes)
            return
        if self.max_own > self.page_columns * page_tokens:
            raise ValueError("Batch: pages has too few columns for max_own")
        if self.prefix_len > (0 if self.tensors[3] is None else self.tensors[3].shape[0]) * page_tokens:
            raise ValueError("Batch: prefix_pages is too short for prefix_len")
        self._checked = page_tokens


class PageStep(NamedTuple):
    """What ``PagePool.step`` found: token_start and own_len are a ``Batch``'s;
    slots and positions are those of the step's tokens."""
    token_start: object
    own_len: object
    n_free: object
    slots: object
    positions: object


class PagePool:
    """The free pages of a cache: ``free`` (int32, one entry per page, device),
    of which the first ``n_free`` (int32, one element, device) are free, the
    next to go out last.  Without tensors: all of n_pages pages, page 0 first."""

    def __init__(self, page_tokens, free=None, n_free=None, n_pages=None, device="cuda"):
        import torch
        if free is None:
            if n_pages is None or n_pages < 1:
                raise ValueError("PagePool: needs the free pages, or how many pages there are")
            free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        if n_free is None:
            n_free = torch.full((1,), free.numel(), dtype=torch.int32, device=free.device)
        for t in (free, n_free):
            if t.dtype != torch.int32 or t.dim() != 1 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("PagePool: free and n_free must be contiguous 1-d int32 CUDA tensors")
        if n_free.numel() != 1:
            raise ValueError("PagePool: n_free has one element")
        self.page_tokens, self.free, self.n_free = page_tokens, free, n_free

    def step(self, own_len, new_len, pages, n_tokens, done=None, prefix_len=0, in_place=True, stream=None):
        """One step's block tables (``sdq_pages_step``): sequences that are
        `done` (int32, may be None) give their pages back, then each gets the
        pages of its new_len new tokens, all of them or none; `pages` (sequences
        x columns, int32) holds the tables.  n_tokens: the rows of the step.
        own_len and the pool's count move on in place, or (in_place=False) stay
        and come back as new tensors."""
        import torch
        i32, n_seqs = torch.int32, own_len.shape[0]
        one, at_own, at_new, at_done = (n_seqs,), own_len.data_ptr(), new_len.data_ptr(), 0
        for t in (own_len, new_len) if done is None else (own_len, new_len, done):
            if t.dtype is not i32 or t.shape != one or not t.is_contiguous() or not t.is_cuda:
                raise ValueError("PagePool.step: own_len, new_len and done must be contiguous int32 CUDA tensors, one element "
                                 "per sequence")
        (rows, columns), (stride, adjacent) = (pages.shape, pages.stride()) if pages.dim() == 2 else ((-1, 0), (0, 0))
        if rows != n_seqs or pages.dtype is not i32 or not pages.is_cuda or (columns > 1 and adjacent != 1):
            raise ValueError("PagePool.step: pages must be an int32 CUDA tensor (sequences, columns), adjacent in a row")
        _check_devices("PagePool.step", own_len, new_len, done, pages, self.free, self.n_free)
        if done is not None:
            at_done = done.data_ptr()
        if in_place and n_seqs > 0 and at_own in (at_new, at_done):
            raise ValueError("PagePool.step: own_len moves on in place and cannot be new_len or done too")
        # one piece of memory: token_start, own_len, the count, slots, positions
        sizes = (n_seqs + 1, n_seqs, 1, n_tokens, n_tokens)
        new = _empty((2 * n_seqs + 2 * n_tokens + 2,), i32, own_len.device, stream)
        start, own_out, n_free, slots, positions = new.split_with_sizes(sizes)
        at, at_free = new.data_ptr(), self.n_free.data_ptr()
        out, out_free = at + 4 * n_seqs + 4, at + 8 * n_seqs + 4
        at_slots, at_positions = out_free + 4, out_free + 4 + 4 * n_tokens
        if in_place:
            own_out, n_free, out, out_free = own_len, self.n_free, at_own, at_free
        sdq_pages_step(_PAGES.pack(self.page_tokens, self.free.shape[0], n_seqs, n_tokens, columns, stride if n_seqs > 1 else columns,
                                   prefix_len, at_own, at_new, at_done, pages.data_ptr(), self.free.data_ptr(), at_free, at, out,
                                   out_free, at_slots, at_positions), stream)
        return PageStep(start, own_out, n_free, slots, positions)


class Rope:
    """Mirror of ``sdq_rope``: cos and sin tables (n_pos x dim / 2, fp32,
    device); ``Rope.table`` makes the usual ones, ``Rope()`` rotates nothing."""

    def __init__(self, cos=None, sin=None, interleaved=False):
        import torch
        if (cos is None) != (sin is None):
            raise ValueError("Rope: cos and sin come together")
        if cos is not None:
            for t in (cos, sin):
                if t.dtype != torch.float32 or t.dim() != 2 or not t.is_cuda or not t.is_contiguous() or t.shape != cos.shape:
                    raise ValueError("Rope: cos and sin must be contiguous 2-d float32 CUDA tensors of one shape")
            if cos.get_device() != sin.get_device():
                raise ValueError("Rope: cos and sin on different devices")
        self.tensors = (cos, sin)
        self.device_index = None if cos is None else cos.get_device()
        self._c = _Rope(_ptr(cos), _ptr(sin), 0 if cos is None else cos.shape[0], 0 if cos is None else 2 * cos.shape[1],
                        int(interleaved))
        self.ref = ctypes.addressof(self._c)

    @classmethod
    def table(cls, n_pos, dim, base=10000.0, interleaved=False, device="cuda"):
        import torch
        cos, sin = sdq_rope_table(n_pos, dim, base)
        return cls(torch.from_numpy(cos).to(device), torch.from_numpy(sin).to(device), interleaved)


class HeadNorm:
    """Mirror of ``sdq_head_norm``: the weights of the heads' norms (fp32,
    device, head_dim of them or heads x head_dim; None: those heads stay)."""

    def __init__(self, q=None, k=None, eps=1e-6):
        import torch
        for t in (q, k):
            if t is not None and (t.dtype != torch.float32 or t.dim() not in (1, 2) or not t.is_cuda or not t.is_contiguous()):
                raise ValueError("HeadNorm: weights must be contiguous float32 CUDA tensors (head_dim) or (heads, head_dim)")
        if not 0 < eps < float("inf"):
            raise ValueError("HeadNorm: eps must be positive and finite")
        self.tensors = (q, k)
        self._c = _HeadNorm(_ptr(q), _ptr(k), int(q is not None and q.dim() == 2), int(k is not None and k.dim() == 2), eps)
        self.ref = ctypes.addressof(self._c)
        self._checked = None

    def check(self, q_heads: int, kv_heads: int, head_dim: int, device):
        """Raise where a weight is not of these heads, or not on this device."""
        if self._checked == (q_heads, kv_heads, head_dim, device):
            return
        for t, heads in zip(self.tensors, (q_heads, kv_heads)):
            if t is not None and tuple(t.shape) not in ((head_dim,), (heads, head_dim)):
                raise ValueError("HeadNorm: weights are not of head_dim, or heads x head_dim, elements")
            if t is not None and t.device != device:
                raise ValueError("HeadNorm: weights on another device than the cache")
        self._checked = q_heads, kv_heads, head_dim, device


class KVCache:
    """Owns an ``sdq_cache`` and holds its two arrays (allocated here, zeroed,
    unless given: bf16, ``desc.shape``, contiguous).  Everything that a call
    works on is on the arrays' device, the current one."""

    device_index = -1   # (of the arrays)

    def __init__(self, desc: CacheDesc, k_pages=None, v_pages=None, device="cuda"):
        import torch
        self.handle = None
        self.desc = desc
        if k_pages is None and v_pages is None:
            k_pages, v_pages = (torch.zeros(desc.shape, dtype=torch.bfloat16, device=device) for _ in range(2))
        for t in (k_pages, v_pages):
            if t is None or t.dtype != torch.bfloat16 or tuple(t.shape) != desc.shape or not t.is_contiguous() or not t.is_cuda:
                raise ValueError("KVCache: both arrays must be contiguous bfloat16 CUDA tensors of desc.shape")
        _check_devices("KVCache", k_pages, v_pages)
        self.k_pages, self.v_pages, self.device_index = k_pages, v_pages, k_pages.get_device()
        self.handle = sdq_cache_create(desc, k_pages, v_pages)

    def close(self):
        if self.handle:
            sdq_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, batch: Batch, q, k, v, rope: Rope, stream=None, norm=None):
        """q, k, v: one row per token (fp32 or bf16; rows may be strided) ->
        the rotated queries (tokens x q_heads x head_dim, bf16); keys and
        values go to the cache.  norm: a HeadNorm, applied to every head of q
        and k ahead of the rotation."""
        import torch
        d, tokens, shape, rows = self.desc, batch.n_tokens, q.shape, k.shape
        dim = d.head_dim
        if len(shape) != 2 or shape[0] != tokens or rows != (tokens, d.kv_heads * dim) or v.shape != rows:
            raise ValueError("KVCache.append: q, k and v need one row of heads x head_dim elements per token")
        (ldq, q1), (ldk, k1), (ldv, v1) = q.stride(), k.stride(), v.stride()
        if not q1 == k1 == v1 == 1:
            raise ValueError("KVCache.append: the elements of a row of q, k and v must be adjacent")
        q_heads, rest = divmod(shape[1], dim)
        if rest:
            raise ValueError("KVCache.append: q's rows are not whole heads")
        if tokens == 1:   # (a single row has no stride of its own)
            ldq, ldk, ldv = shape[1], rows[1], rows[1]
        batch.check(d.page_tokens)
        at = self.device_index
        if not q.get_device() == k.get_device() == v.get_device() == batch.device_index == at or rope.device_index not in (None, at):
            raise ValueError("KVCache.append: q, k, v, the batch and the rotation tables must be on the cache's device")
        if norm is not None:
            norm.check(q_heads, d.kv_heads, dim, self.k_pages.device)
        kind = q.dtype
        kind = -1 if k.dtype is not kind or v.dtype is not kind else SDQ_F32 if kind is torch.float32 else SDQ_BF16 if kind is torch.bfloat16 else -1
        out = _empty((tokens, q_heads, dim), torch.bfloat16, q.device, stream)
        if norm is None:
            _check(lib().sdq_cache_append(self.handle, batch.ref, q_heads, q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                          kind, rope.ref, out.data_ptr(), _stream(stream)), "sdq_cache_append")
        else:
            _check(lib().sdq_cache_append_norm(self.handle, batch.ref, q_heads, q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(),
                                               ldv, kind, rope.ref, norm.ref, out.data_ptr(), _stream(stream)),
                   "sdq_cache_append_norm")
        return out

    def alloc_workspace(self, batch: Batch, q_heads: int, stream=None, window=None, sinks=0):
        """For ``attend`` on this batch (or one of the same integers) with this window."""
        import torch
        if window is None:
            n = sdq_attention_workspace_bytes(self.handle, batch, q_heads)
        else:
            n = sdq_attention_window_workspace_bytes(self.handle, batch, q_heads, window, sinks)
        if n == 0:
            raise SdqError(-1, "sdq_attention_workspace_bytes" if window is None else "sdq_attention_window_workspace_bytes")
        return _empty(n, torch.uint8, self.k_pages.device, stream)

    def attend(self, batch: Batch, q, scale=None, ws=None, lse=None, stream=None, window=None, sinks=0):
        """q (tokens x q_heads x head_dim, bf16; tokens may be strided) ->
        outputs of the same shape in bf16.  scale: 1 / sqrt(head_dim) unless
        given; lse: fp32 (tokens x q_heads), written if given.  window: a token
        sees that many positions up to its own, and the first `sinks` ones
        (positions count the prefix); None: all of them."""
        import torch
        d, tokens, dim, shape = self.desc, batch.n_tokens, self.desc.head_dim, q.shape
        if len(shape) != 3 or shape[0] != tokens or shape[2] != dim or q.dtype != torch.bfloat16 or not q.is_cuda:
            raise ValueError("KVCache.attend: q must be a bfloat16 CUDA tensor (tokens, q_heads, head_dim)")
        heads, stride = shape[1], q.stride()
        if stride[2] != 1 or (heads > 1 and stride[1] != dim):
            raise ValueError("KVCache.attend: the heads of a token of q must be adjacent")
        if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (tokens, heads)
                                or not lse.is_contiguous() or not lse.is_cuda):
            raise ValueError("KVCache.attend: lse must be a contiguous float32 CUDA tensor (tokens, q_heads)")
        if window is None and sinks != 0:
            raise ValueError("KVCache.attend: sinks belong to a window")
        batch.check(d.page_tokens)
        at = self.device_index
        if not q.get_device() == batch.device_index == at or (lse is not None and lse.get_device() != at):
            raise ValueError("KVCache.attend: q, the batch and lse must be on the cache's device")
        if ws is None:
            ws = self.alloc_workspace(batch, heads, stream, window, sinks)
        elif not ws.is_cuda or not ws.is_contiguous() or ws.get_device() != at:
            raise ValueError("KVCache.attend: ws must be a contiguous CUDA tensor on the cache's device")
        out = _empty((tokens, heads, dim), torch.bfloat16, q.device, stream)
        ldq, scale = stride[0] if tokens > 1 else heads * dim, dim ** -0.5 if scale is None else scale
        if window is None:
            sdq_attention(self.handle, batch, heads, q, ldq, scale, out, lse, ws, stream)
        else:
            sdq_attention_window(self.handle, batch, heads, q, ldq, scale, window, sinks, out, lse, ws, stream)
        return out


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """One token per row of logits (rows x vocab, fp32 or bf16; rows may be
    strided) from one random number per row -> int32 tokens.  The settings:
    one per row (float32, top_k int32), or None for none."""
    import torch
    shape = logits.shape
    if len(shape) != 2 or logits.stride()[1] != 1 or not logits.is_cuda:
        raise ValueError("sample: logits must be a CUDA tensor (rows, vocab) with adjacent elements in a row")
    rows, f32 = shape[:1], torch.float32
    _check_devices("sample", logits)
    at = logits.get_device()
    for t, dtype in ((u, f32), (temperature, f32), (top_k, torch.int32), (top_p, f32), (min_p, f32)):
        if t is not None and (t.dtype is not dtype or t.shape != rows or not t.is_contiguous() or t.get_device() != at):
            raise ValueError("sample: u, temperature, top_p and min_p are float32, top_k int32, one per row, on the logits' GPU")
    tokens = _empty(rows, torch.int32, logits.device, stream)
    sdq_sample(logits, u, temperature, top_k, top_p, min_p, tokens, stream)
    return tokens


def adjust_logits(logits, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias=None, allowed=None, allowed_row=None, out=None, stream=None):
    """Penalties for repeated tokens, biases and a grammar's allowed tokens on
    logits (rows x vocab, fp32 or bf16; rows may be strided) -> logits of the
    same type, in ``out`` if given (may be ``logits``).  history (rows x places,
    int32; rows may be strided) holds each row's tokens so far, of which
    history_len count (None: all) and prompt_len are the prompt's (None: 0);
    repetition, frequency, presence: float32, one per row.  bias_ids (int32,
    negative: unused) and bias (float32): rows x entries.  allowed (int32 words
    of 32 tokens, sets x ceil(vocab / 32)), allowed_row: the set of each row
    (int32, -1 for none; None: row i has set i)."""
    import torch
    shape, i32, f32 = logits.shape, torch.int32, torch.float32
    if len(shape) != 2 or logits.stride()[1] != 1 or not logits.is_cuda:
        raise ValueError("adjust_logits: logits must be a CUDA tensor (rows, vocab) with adjacent elements in a row")
    rows, vocab = shape
    one = (rows,)

    def per_row(t, dtype):
        if t is None:
            return 0
        if t.dtype is not dtype or t.shape != one or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("adjust_logits: repetition, frequency and presence are float32, history_len, prompt_len and "
                             "allowed_row int32, one per row, on the GPU")
        return t.data_ptr()

    def table(t, dtype, n):
        if t is None:
            return 0, 0, 0
        columns, stride = t.shape, t.stride()
        if (t.dtype is not dtype or len(columns) != 2 or not t.is_cuda or (n is not None and columns[0] != n)
                or (columns[1] > 1 and stride[1] != 1)):
            raise ValueError("adjust_logits: history, bias_ids and bias need one row for each of logits, allowed one for each "
                             "set: 2-d CUDA tensors, int32 (bias: float32), adjacent in a row")
        return t.data_ptr(), stride[0], columns[1]

    at_history, ld_history, places = table(history, i32, rows)
    at_ids, ld_ids, n_ids = table(bias_ids, i32, rows)
    at_bias, ld_bias, n_bias = table(bias, f32, rows)
    at_allowed, ld_allowed, words = table(allowed, i32, None)
    if (bias_ids is None) != (bias is None) or n_ids != n_bias:
        raise ValueError("adjust_logits: bias_ids and bias come together, of one shape")
    if history is None and (history_len is not None or prompt_len is not None):
        raise ValueError("adjust_logits: history_len and prompt_len belong to a history")
    if allowed is None and allowed_row is not None:
        raise ValueError("adjust_logits: allowed_row belongs to allowed")
    if allowed is not None and words < (vocab + 31) // 32:
        raise ValueError("adjust_logits: the sets of allowed have too few words")
    if allowed is not None and at_allowed == 0 and allowed_row is None:   # (no memory: as if it were not given)
        raise ValueError("adjust_logits: allowed needs a set for each row, or allowed_row")
    _check_devices("adjust_logits", logits, history, history_len, prompt_len, repetition, frequency, presence, bias_ids, bias,
                   allowed, allowed_row, out)
    if out is None:
        out = _empty(shape, logits.dtype, logits.device, stream)
    elif out.shape != shape or out.dtype is not logits.dtype or out.stride()[1] != 1 or not out.is_cuda:
        raise ValueError("adjust_logits: out must be like logits")
    a = _ADJUST.pack(at_history, per_row(history_len, i32), per_row(prompt_len, i32), per_row(repetition, f32),
                     per_row(frequency, f32), per_row(presence, f32), at_ids, at_bias, at_allowed, per_row(allowed_row, i32),
                     ld_history, ld_ids, ld_bias, ld_allowed, places, n_bias, 0 if allowed is None else allowed.shape[0])
    sdq_adjust_logits(logits, a, out, stream)
    return out
