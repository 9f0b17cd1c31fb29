"""ctypes binding of the C ABI declared in include/dfss.h.

Each function has the name of the C entry point it calls (dfss_attention_ragged
calls its _split form where that is the faster one) and only marshals arguments:
tensors are passed as raw device pointers, the current PyTorch HIP stream as the
stream handle, and arrays that are not given are allocated.  There is no fallback: if ``libdfss.so`` is
missing or a call reports an error, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass, fields
from functools import cached_property
from operator import attrgetter

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdfss.so")

EXPORTS = (
    "dfss_vals_bytes", "dfss_meta_bytes", "dfss_workspace_bytes", "dense_workspace_bytes",
    "dfss_sddmm_prune", "dfss_sparse_softmax", "dfss_spmm", "dfss_attention", "dense_attention",
    "dense_attention_fused", "dfss_meta_to_canonical", "dfss_meta_from_canonical", "dfss_status_string",
    "dfss_sddmm_prune_bias", "dfss_attention_bias", "dense_attention_bias", "dense_attention_fused_bias",
    "dfss_attention_blocked", "dense_attention_fused_blocked", "dfss_spmm_t",
    "dfss_backward_workspace_bytes", "dfss_attention_backward",
    "dfss_attention_ragged", "dense_attention_fused_ragged",
    "dfss_attention_staged", "dfss_attention_staged_bias",
    "dfss_static_scratch_bytes", "dfss_attention_staged_static",
    "dfss_sddmm_prune_causal", "dfss_attention_causal", "dfss_attention_staged_causal", "dense_attention_causal",
    "dense_attention_fused_causal",
    "dfss_blocked_split_workspace_bytes", "dfss_attention_blocked_split", "dense_attention_fused_blocked_split",
    "dfss_sddmm_prune_mask", "dfss_attention_staged_mask", "dense_attention_mask",
    "dfss_attention_mask", "dense_attention_fused_mask",
    "dfss_attention_varlen",
    "dfss_ragged_split_workspace_bytes", "dfss_attention_ragged_split",
    "dfss_qk_norm_rotate", "dfss_qk_norm_workspace_bytes", "dfss_qk_norm_rotate_backward",
    "dfss_cache_append", "dfss_cached_workspace_bytes", "dfss_attention_cached", "dense_attention_cached",
)
# exported for the library's own tests only (csrc/dfss_internal.h)
INTERNAL_EXPORTS = ("dfss_internal_attention_variant", "dfss_internal_norm_plan", "dfss_internal_append_plan", "dfss_internal_cached_plan")
VARIANT_AUTO, VARIANT_Q16, VARIANT_Q16X2, VARIANT_Q32W2, VARIANT_Q32W4, VARIANT_Q32K2, VARIANT_FEW = range(7)


DFSS_BF16, DFSS_F32, DFSS_F32_BF16X3 = 0, 1, 2


class DfssError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn} failed: status {status} ({text})")
        self.status = status


class _CShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "Lq", "Lk", "d", "N", "M", "dtype")]


# dfss_rows, dfss_rotary, dfss_cache as bytes (a ctypes structure takes 2 us to fill, more than the checks of its tensors)
_ROWS = struct.Struct("@Piqqq")
_ROTARY = struct.Struct("@PPPiii")
_CACHE = struct.Struct("@PPPPPPiiii")


class _Call:
    """Element types, sizes and the C structure of a shape, as the calls use them.  (Deriving them on every call took 4 of
    the 11 us of host time of a small one, as much as the kernel launch itself.)"""
    __slots__ = ("c", "ref", "torch_dtype", "O_shape", "q_numel", "kv_numel", "ragged_ws", "cached_ws")

    def __init__(self, s: Shape):
        self.c = s.c()
        self.ref = ctypes.byref(self.c)     # read by the C side only
        self.torch_dtype = s.torch_dtype
        self.O_shape = (s.BH, s.Lq, s.d)
        self.q_numel = s.BH * s.Lq * s.d
        self.kv_numel = s.BH * s.Lk * s.d
        self.ragged_ws = None               # workspace bytes of dfss_attention_ragged, asked for once
        self.cached_ws = {}                 # ... of the calls over a cache, by its heads


@dataclass(frozen=True)
class Shape:
    """Mirror of ``dfss_shape``: B*H heads, Lq queries, Lk keys, head size d, keep N of M."""
    B: int
    H: int
    Lq: int
    Lk: int
    d: int
    N: int = 2
    M: int = 4
    dtype: int = 0  # DFSS_BF16 = 0; DFSS_F32 = 1, DFSS_F32_BF16X3 = 2 (the 4-byte mode: 1:2 only)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == DFSS_BF16 else torch.float32

    @property
    def LqP(self) -> int:
        """Rows of the compressed arrays (vals, meta, the dense workspace): Lq, rounded up to a multiple of 64 where
        the stage calls take an unpadded length (2-byte dtype)."""
        return (self.Lq + 63) // 64 * 64

    @property
    def LkP(self) -> int:
        """Keys of the compressed arrays: Lk, rounded up to a multiple of 128 where the stage calls take an unpadded
        length."""
        return (self.Lk + 127) // 128 * 128

    @property
    def meta_words(self) -> int:
        """uint16 metadata words per row: one 4-bit code per 8 bytes of dense data."""
        return self.LkP // (16 if self.dtype == DFSS_BF16 else 8)

    def c(self) -> _CShape:
        return _CShape(self.B, self.H, self.Lq, self.Lk, self.d, self.N, self.M, self.dtype)

    @cached_property
    def _call(self) -> _Call:
        """What every call with this shape needs, derived once (a function of the fields, which do not change)."""
        return _Call(self)

    def __getstate__(self):   # copies and pickles carry the fields only
        return {f.name: getattr(self, f.name) for f in fields(self)}

    @property
    def BH(self) -> int:
        return self.B * self.H

    @property
    def Lc(self) -> int:
        """Kept entries per row of the compressed arrays."""
        return self.LkP * self.N // self.M


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libdfss.so (built in-tree by ``paper_2203_00091_amd.build``); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} not built: run `python -m paper_2203_00091_amd.build` (needs hipcc)")
        L = ctypes.CDLL(_LIB_PATH)
        sp = ctypes.POINTER(_CShape)
        vp, sz, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
        for name in ("dfss_vals_bytes", "dfss_meta_bytes", "dfss_workspace_bytes", "dense_workspace_bytes",
                     "dfss_backward_workspace_bytes", "dfss_blocked_split_workspace_bytes",
                     "dfss_ragged_split_workspace_bytes"):
            getattr(L, name).argtypes = [sp]
            getattr(L, name).restype = sz
        L.dfss_sddmm_prune.argtypes = [vp, vp, sp, f32, vp, vp, vp]
        L.dfss_sparse_softmax.argtypes = [vp, sp, vp]
        L.dfss_spmm.argtypes = [vp, vp, vp, sp, vp, vp]
        L.dfss_attention.argtypes = [vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention.argtypes = [vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_fused.argtypes = [vp, vp, vp, sp, f32, vp, vp]
        L.dfss_sddmm_prune_bias.argtypes = [vp, vp, vp, sp, f32, vp, vp, vp]
        L.dfss_attention_bias.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_bias.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_fused_bias.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_blocked.argtypes = [vp, vp, vp, vp, vp, sp, f32, vp, vp]
        L.dense_attention_fused_blocked.argtypes = [vp, vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_blocked_split.argtypes = [vp, vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_fused_blocked_split.argtypes = [vp, vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dfss_sddmm_prune_mask.argtypes = [vp, vp, vp, sp, f32, vp, vp, vp]
        L.dfss_attention_staged_mask.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_mask.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dfss_attention_mask.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_varlen.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dense_attention_fused_mask.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_ragged.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_ragged_split.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dfss_attention_staged.argtypes = [vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dfss_attention_staged_bias.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dfss_attention_staged_static.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_sddmm_prune_causal.argtypes = [vp, vp, vp, sp, f32, vp, vp, vp]
        L.dfss_attention_causal.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_staged_causal.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_causal.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp, sz, vp]
        L.dense_attention_fused_causal.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_attention_staged_static.restype = ctypes.c_int
        L.dfss_static_scratch_bytes.argtypes = []
        L.dfss_static_scratch_bytes.restype = sz
        L.dfss_internal_attention_variant.argtypes = [vp, vp, vp, vp, sp, f32, vp, ctypes.c_int, ctypes.c_int, vp]
        L.dense_attention_fused_ragged.argtypes = [vp, vp, vp, vp, sp, f32, vp, vp]
        L.dfss_spmm_t.argtypes = [vp, vp, vp, sp, vp, vp]
        L.dfss_attention_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, sp, f32, vp, vp, vp, vp, sz, vp]
        L.dfss_meta_to_canonical.argtypes = [vp, sp, vp, vp]
        L.dfss_meta_from_canonical.argtypes = [vp, sp, vp, vp]
        rows = rot = cache = vp     # (given as bytes)
        n32 = ctypes.c_int32
        L.dfss_qk_norm_rotate.argtypes = [rows, rows, vp, vp, rot, sp, f32, rows, rows, vp]
        L.dfss_qk_norm_workspace_bytes.argtypes = [sp]
        L.dfss_qk_norm_workspace_bytes.restype = sz
        L.dfss_qk_norm_rotate_backward.argtypes = [rows, rows, rows, rows, vp, vp, rot, sp, f32, rows, rows, vp, vp, vp, sz, vp]
        L.dfss_cache_append.argtypes = [rows, rows, n32, vp, cache, vp, rot, sp, f32, vp]
        L.dfss_cached_workspace_bytes.argtypes = [sp, cache]
        L.dfss_cached_workspace_bytes.restype = sz
        L.dfss_attention_cached.argtypes = [rows, n32, vp, cache, sp, f32, n32, vp, vp, sz, vp]
        L.dense_attention_cached.argtypes = [rows, n32, vp, cache, sp, f32, n32, vp, vp, sz, vp]
        for name in ("dfss_qk_norm_rotate", "dfss_qk_norm_rotate_backward", "dfss_cache_append", "dfss_attention_cached",
                     "dense_attention_cached"):
            getattr(L, name).restype = ctypes.c_int
        for name in ("dfss_sddmm_prune", "dfss_sparse_softmax", "dfss_spmm", "dfss_attention",
                     "dense_attention", "dense_attention_fused", "dfss_meta_to_canonical", "dfss_meta_from_canonical",
                     "dfss_sddmm_prune_bias", "dfss_attention_bias", "dense_attention_bias",
                     "dense_attention_fused_bias", "dfss_attention_blocked", "dense_attention_fused_blocked",
                     "dfss_attention_ragged", "dense_attention_fused_ragged", "dfss_spmm_t",
                     "dfss_attention_backward", "dfss_attention_staged", "dfss_attention_staged_bias",
                     "dfss_internal_attention_variant", "dfss_sddmm_prune_causal", "dfss_attention_causal",
                     "dfss_attention_staged_causal", "dense_attention_causal", "dense_attention_fused_causal",
                     "dfss_attention_blocked_split", "dense_attention_fused_blocked_split",
                     "dfss_sddmm_prune_mask", "dfss_attention_staged_mask", "dense_attention_mask",
                     "dfss_attention_mask", "dense_attention_fused_mask",
                     "dfss_attention_varlen", "dfss_attention_ragged_split"):
            getattr(L, name).restype = ctypes.c_int
        L.dfss_status_string.argtypes = [ctypes.c_int]
        L.dfss_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(fn: str, status: int):
    if status != 0:
        raise DfssError(fn, status, load_library().dfss_status_string(status).decode())


def _stream() -> int:
    """Handle of the current stream of the current device (without the Stream object around it: 2.7 us a call).  Called
    after the tensors' checks, so that the runtime is up."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t: torch.Tensor | None) -> int | None:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


def _data(t: torch.Tensor | None, s: Shape, *shape) -> int | None:
    """Pointer of a Q/K/V/O/vals-like tensor after checking that its element type is the one the shape
    declares and its size the one the call will touch (the C side sees raw pointers only)."""
    if t is None:
        return None
    if t.dtype != s.torch_dtype:
        raise ValueError(f"expected a {s.torch_dtype} tensor for dfss_shape.dtype = {s.dtype}, got {t.dtype}")
    n = 1
    for k in shape:
        n *= k
    if t.numel() != n:
        raise ValueError(f"expected {n} elements {shape}, got {t.numel()}")
    return _ptr(t)


def _q(t, s: Shape):      # Q, O and their gradients: [BH, Lq, d]
    c = s._call
    if t is not None and t.dtype is c.torch_dtype and t.numel() == c.q_numel and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    return _data(t, s, s.BH, s.Lq, s.d)


def _kv(t, s: Shape):     # K, V and their gradients: [BH, Lk, d]
    c = s._call
    if t is not None and t.dtype is c.torch_dtype and t.numel() == c.kv_numel and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    return _data(t, s, s.BH, s.Lk, s.d)


def _kept(t, s: Shape):   # kept scores / weights: [BH, Lq, Lk*N/M]
    return _data(t, s, s.BH, s.LqP, s.Lc)


def _meta(t: torch.Tensor, s: Shape) -> int:
    if t.element_size() != 2 or t.numel() != s.BH * s.LqP * s.meta_words:
        raise ValueError(f"metadata must hold {s.BH * s.LqP * s.meta_words} 16-bit words")
    return _ptr(t)


def dfss_vals_bytes(s: Shape) -> int:
    return int(load_library().dfss_vals_bytes(s._call.ref))


def dfss_meta_bytes(s: Shape) -> int:
    return int(load_library().dfss_meta_bytes(s._call.ref))


def dfss_workspace_bytes(s: Shape) -> int:
    return int(load_library().dfss_workspace_bytes(s._call.ref))


def dense_workspace_bytes(s: Shape) -> int:
    return int(load_library().dense_workspace_bytes(s._call.ref))


def _alloc_bytes(n: int, device) -> torch.Tensor:
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def dfss_sddmm_prune(Q, K, s: Shape, scale: float, vals=None, meta=None):
    """Stage 1.  Returns (vals [BH, Lq, Lk*N/M] in the shape's dtype, meta: 16-bit words in library order)."""
    if vals is None:
        vals = torch.empty((s.BH, s.LqP, s.Lc), dtype=s.torch_dtype, device=Q.device)
    if meta is None:
        meta = torch.empty((s.BH * s.LqP * s.meta_words,), dtype=torch.int16, device=Q.device)
    st = load_library().dfss_sddmm_prune(_q(Q, s), _kv(K, s), s._call.ref, scale,
                                         _kept(vals, s), _meta(meta, s), _stream())
    _check("dfss_sddmm_prune", st)
    return vals, meta


def dfss_sparse_softmax(vals, s: Shape):
    """Stage 2, in place on vals."""
    _check("dfss_sparse_softmax", load_library().dfss_sparse_softmax(_kept(vals, s), s._call.ref, _stream()))
    return vals


def dfss_spmm(vals, meta, V, s: Shape, O=None):
    """Stage 3.  Returns O [BH, Lq, d]."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=V.device)
    st = load_library().dfss_spmm(_kept(vals, s), _meta(meta, s), _kv(V, s),
                                  s._call.ref, _q(O, s), _stream())
    _check("dfss_spmm", st)
    return O


def _needs_workspace(s: Shape) -> bool:
    """Only the exact-product float mode runs dfss_attention through a workspace."""
    return s.dtype == DFSS_F32


def dfss_attention(Q, K, V, s: Shape, scale: float, O=None, ws=None):
    """Whole DFSS forward in one kernel.  ``ws`` is passed on if given (the library uses it with DFSS_F32 only,
    where it is allocated here if absent)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None and _needs_workspace(s):
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention(_q(Q, s), _kv(K, s), _kv(V, s),
                                       s._call.ref, scale, _q(O, s), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention", st)
    return O


def dfss_attention_staged(Q, K, V, s: Shape, scale: float, O=None, ws=None):
    """Whole DFSS forward through ``ws`` (allocated if not given): stage 1, then the product that applies the
    softmax as it reads the kept scores (4-byte dtypes: the three stage kernels)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_staged(_q(Q, s), _kv(K, s), _kv(V, s),
                                              s._call.ref, scale, _q(O, s), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_staged", st)
    return O


def dfss_attention_staged_bias(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """dfss_attention_staged with an additive key bias (may be None)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_staged_bias(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                   s._call.ref, scale, _q(O, s), _ptr(ws),
                                                   ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_staged_bias", st)
    return O


def dfss_static_scratch_bytes() -> int:
    return int(load_library().dfss_static_scratch_bytes())


def dfss_attention_staged_static(Q, K, V, key_bias, s: Shape, scale: float, O):
    """The staged forward pass with the library's own fixed scratch array; allocates nothing (O is the caller's)."""
    st = load_library().dfss_attention_staged_static(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                     s._call.ref, scale, _q(O, s), _stream())
    _check("dfss_attention_staged_static", st)
    return O


def internal_attention_variant(Q, K, V, key_bias, s: Shape, scale: float, variant: int, dense: bool = False, O=None):
    """Test hook: the one-kernel forward pass (DFSS, or full attention if ``dense``) with a named tiling."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_internal_attention_variant(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                        s._call.ref, scale, _q(O, s), int(variant),
                                                        int(bool(dense)), _stream())
    _check("dfss_internal_attention_variant", st)
    return O


def dense_attention(Q, K, V, s: Shape, scale: float, O=None, ws=None):
    """Full attention baseline on the same GPU."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dense_workspace_bytes(s), Q.device)
    st = load_library().dense_attention(_q(Q, s), _kv(K, s), _kv(V, s),
                                        s._call.ref, scale, _q(O, s), _ptr(ws),
                                        ws.numel() * ws.element_size(), _stream())
    _check("dense_attention", st)
    return O


def dense_attention_fused(Q, K, V, s: Shape, scale: float, O=None):
    """Full attention in one kernel (the stronger baseline)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused(_q(Q, s), _kv(K, s), _kv(V, s),
                                              s._call.ref, scale, _q(O, s),
                                              _stream())
    _check("dense_attention_fused", st)
    return O


def _bias_ptr(key_bias, s: Shape):
    if key_bias is None:
        return None
    if key_bias.dtype != torch.float32 or tuple(key_bias.shape) != (s.B, s.Lk):
        raise ValueError(f"key_bias must be float32 [B, Lk] = [{s.B}, {s.Lk}]")
    return _ptr(key_bias)


def dfss_sddmm_prune_bias(Q, K, key_bias, s: Shape, scale: float, vals=None, meta=None):
    """Stage 1 with an additive key bias (float32 [B, Lk] device tensor, -inf masks a key)."""
    if vals is None:
        vals = torch.empty((s.BH, s.LqP, s.Lc), dtype=s.torch_dtype, device=Q.device)
    if meta is None:
        meta = torch.empty((s.BH * s.LqP * s.meta_words,), dtype=torch.int16, device=Q.device)
    st = load_library().dfss_sddmm_prune_bias(_q(Q, s), _kv(K, s), _bias_ptr(key_bias, s),
                                              s._call.ref, scale, _kept(vals, s), _meta(meta, s), _stream())
    _check("dfss_sddmm_prune_bias", st)
    return vals, meta


def dfss_attention_bias(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """Whole DFSS forward (one kernel) with an additive key bias."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None and _needs_workspace(s):
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_bias(_q(Q, s), _kv(K, s), _kv(V, s),
                                            _bias_ptr(key_bias, s), s._call.ref, scale, _q(O, s), _ptr(ws),
                                            0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_bias", st)
    return O


def dense_attention_bias(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """Full attention (three stages) with an additive key bias."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dense_workspace_bytes(s), Q.device)
    st = load_library().dense_attention_bias(_q(Q, s), _kv(K, s), _kv(V, s),
                                             _bias_ptr(key_bias, s), s._call.ref, scale, _q(O, s), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream())
    _check("dense_attention_bias", st)
    return O


def dense_attention_fused_bias(Q, K, V, key_bias, s: Shape, scale: float, O=None):
    """Full attention in one kernel with an additive key bias."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused_bias(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                   s._call.ref, scale, _q(O, s), _stream())
    _check("dense_attention_fused_bias", st)
    return O


def dfss_sddmm_prune_causal(Q, K, key_bias, s: Shape, scale: float, vals=None, meta=None):
    """Stage 1 under the causal mask (query i sees keys 0 .. i + Lk - Lq); key_bias may be None."""
    if vals is None:
        vals = torch.empty((s.BH, s.LqP, s.Lc), dtype=s.torch_dtype, device=Q.device)
    if meta is None:
        meta = torch.empty((s.BH * s.LqP * s.meta_words,), dtype=torch.int16, device=Q.device)
    st = load_library().dfss_sddmm_prune_causal(_q(Q, s), _kv(K, s), _bias_ptr(key_bias, s),
                                                s._call.ref, scale, _kept(vals, s), _meta(meta, s), _stream())
    _check("dfss_sddmm_prune_causal", st)
    return vals, meta


def dfss_attention_causal(Q, K, V, key_bias, s: Shape, scale: float, O=None):
    """Whole DFSS forward in one kernel under the causal mask; key_bias may be None."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_attention_causal(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                              s._call.ref, scale, _q(O, s), _stream())
    _check("dfss_attention_causal", st)
    return O


def dfss_attention_staged_causal(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """dfss_attention_staged under the causal mask; key_bias may be None."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_staged_causal(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                     s._call.ref, scale, _q(O, s), _ptr(ws),
                                                     ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_staged_causal", st)
    return O


def dense_attention_causal(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """Full attention (three stages) under the causal mask; key_bias may be None."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dense_workspace_bytes(s), Q.device)
    st = load_library().dense_attention_causal(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                               s._call.ref, scale, _q(O, s), _ptr(ws),
                                               ws.numel() * ws.element_size(), _stream())
    _check("dense_attention_causal", st)
    return O


def dense_attention_fused_causal(Q, K, V, key_bias, s: Shape, scale: float, O=None):
    """Full attention in one kernel under the causal mask; key_bias may be None."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused_causal(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                     s._call.ref, scale, _q(O, s), _stream())
    _check("dense_attention_fused_causal", st)
    return O


def dfss_attention_ragged(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """DFSS forward on unpadded arrays: any Lq, Lk a multiple of 4; key_bias may be None.  One kernel, except for few queries
    against many keys without a key bias (dfss_ragged_split_workspace_bytes is not 0): those calls are
    dfss_attention_ragged_split, with ``ws`` as described there.  Elsewhere ``ws`` is not touched."""
    n = s._call.ragged_ws
    if n is None:
        n = s._call.ragged_ws = dfss_ragged_split_workspace_bytes(s)
    if n and key_bias is None:
        return dfss_attention_ragged_split(Q, K, V, None, s, scale, O, ws)
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_attention_ragged(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                              s._call.ref, scale, _q(O, s), _stream())
    _check("dfss_attention_ragged", st)
    return O


def dfss_attention_ragged_split(Q, K, V, key_bias, s: Shape, scale: float, O=None, ws=None):
    """dfss_attention_ragged with a workspace of dfss_ragged_split_workspace_bytes (allocated if not given), through which
    several workgroups share the keys of a query tile: two kernels."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        n = dfss_ragged_split_workspace_bytes(s) if key_bias is None else 0
        if n:
            ws = _alloc_bytes(n, Q.device)
    st = load_library().dfss_attention_ragged_split(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                    s._call.ref, scale, _q(O, s), _ptr(ws),
                                                    0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_ragged_split", st)
    return O


def dfss_ragged_split_workspace_bytes(s: Shape) -> int:
    return int(load_library().dfss_ragged_split_workspace_bytes(s._call.ref))


def dense_attention_fused_ragged(Q, K, V, key_bias, s: Shape, scale: float, O=None):
    """Full attention in one kernel on unpadded arrays (the baseline of dfss_attention_ragged)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused_ragged(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                     s._call.ref, scale, _q(O, s), _stream())
    _check("dense_attention_fused_ragged", st)
    return O


def _block_mask_ptr(block_mask, s: Shape):
    if block_mask.dtype != torch.uint8 or tuple(block_mask.shape) != (s.Lq // 64, s.Lk // 64):
        raise ValueError(f"block_mask must be uint8 [Lq/64, Lk/64] = [{s.Lq // 64}, {s.Lk // 64}]")
    return _ptr(block_mask)


def dfss_attention_blocked(Q, K, V, key_bias, block_mask, s: Shape, scale: float, O=None):
    """DFSS forward restricted to the 64 x 64 score blocks with a non-zero entry in block_mask."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_attention_blocked(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                               _block_mask_ptr(block_mask, s), s._call.ref, scale, _q(O, s),
                                               _stream())
    _check("dfss_attention_blocked", st)
    return O


def dense_attention_fused_blocked(Q, K, V, key_bias, block_mask, s: Shape, scale: float, O=None):
    """Block-sparse full attention (same block pattern, no N:M pruning)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused_blocked(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                      _block_mask_ptr(block_mask, s), s._call.ref, scale,
                                                      _q(O, s), _stream())
    _check("dense_attention_fused_blocked", st)
    return O


def _mask_ptr(mask: torch.Tensor, s: Shape) -> int:
    if mask.dtype != torch.float32 or mask.numel() != s.Lq * s.Lk:
        raise ValueError(f"the mask must be float32 [{s.Lq}, {s.Lk}]")
    return _ptr(mask)


def dfss_sddmm_prune_mask(Q, K, mask, s: Shape, scale: float, vals=None, meta=None):
    """Stage 1 with an additive mask [Lq, Lk] shared by all heads."""
    if vals is None:
        vals = torch.empty((s.BH, s.LqP, s.Lc), dtype=s.torch_dtype, device=Q.device)
    if meta is None:
        meta = torch.empty((s.BH * s.LqP * s.meta_words,), dtype=torch.int16, device=Q.device)
    st = load_library().dfss_sddmm_prune_mask(_q(Q, s), _kv(K, s), _mask_ptr(mask, s), s._call.ref, scale,
                                              _kept(vals, s), _meta(meta, s), _stream())
    _check("dfss_sddmm_prune_mask", st)
    return vals, meta


def dfss_attention_staged_mask(Q, K, V, mask, s: Shape, scale: float, O=None, ws=None):
    """dfss_attention_staged with an additive mask [Lq, Lk] shared by all heads."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_staged_mask(_q(Q, s), _kv(K, s), _kv(V, s), _mask_ptr(mask, s),
                                                   s._call.ref, scale, _q(O, s), _ptr(ws),
                                                   ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_staged_mask", st)
    return O


def dense_attention_mask(Q, K, V, mask, s: Shape, scale: float, O=None, ws=None):
    """Full attention (three kernels) with the same mask."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dense_workspace_bytes(s), Q.device)
    st = load_library().dense_attention_mask(_q(Q, s), _kv(K, s), _kv(V, s), _mask_ptr(mask, s), s._call.ref,
                                             scale, _q(O, s), _ptr(ws), ws.numel() * ws.element_size(), _stream())
    _check("dense_attention_mask", st)
    return O


def _len_ptr(key_len: torch.Tensor, s: Shape) -> int:
    if key_len.dtype != torch.int32 or key_len.numel() != s.B:
        raise ValueError(f"key_len must be int32 [B] = [{s.B}]")
    return _ptr(key_len)


def dfss_attention_varlen(Q, K, V, key_len, s: Shape, scale: float, O=None):
    """DFSS forward in one kernel on a padded batch: keys key_len[b] .. Lk - 1 of batch element b are padding."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_attention_varlen(_q(Q, s), _kv(K, s), _kv(V, s), _len_ptr(key_len, s), s._call.ref,
                                              scale, _q(O, s), _stream())
    _check("dfss_attention_varlen", st)
    return O


def dfss_attention_mask(Q, K, V, mask, s: Shape, scale: float, O=None):
    """DFSS forward in one kernel with an additive mask fp32 [Lq, Lk] (any Lq, Lk a multiple of 4; arrays unpadded)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dfss_attention_mask(_q(Q, s), _kv(K, s), _kv(V, s), _mask_ptr(mask, s), s._call.ref,
                                            scale, _q(O, s), _stream())
    _check("dfss_attention_mask", st)
    return O


def dense_attention_fused_mask(Q, K, V, mask, s: Shape, scale: float, O=None):
    """Full attention in one kernel with the same mask (the baseline of dfss_attention_mask)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    st = load_library().dense_attention_fused_mask(_q(Q, s), _kv(K, s), _kv(V, s), _mask_ptr(mask, s),
                                                   s._call.ref, scale, _q(O, s), _stream())
    _check("dense_attention_fused_mask", st)
    return O


def dfss_blocked_split_workspace_bytes(s: Shape) -> int:
    return int(load_library().dfss_blocked_split_workspace_bytes(s._call.ref))


def dfss_attention_blocked_split(Q, K, V, key_bias, block_mask, s: Shape, scale: float, O=None, ws=None):
    """dfss_attention_blocked with a workspace: long row blocks are shared between several workgroups."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_blocked_split_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_blocked_split(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                     _block_mask_ptr(block_mask, s), s._call.ref, scale,
                                                     _q(O, s), ws.data_ptr(), ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_blocked_split", st)
    return O


def dense_attention_fused_blocked_split(Q, K, V, key_bias, block_mask, s: Shape, scale: float, O=None, ws=None):
    """Block-sparse full attention with the same workspace (the baseline of dfss_attention_blocked_split)."""
    if O is None:
        O = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_blocked_split_workspace_bytes(s), Q.device)
    st = load_library().dense_attention_fused_blocked_split(_q(Q, s), _kv(K, s), _kv(V, s), _bias_ptr(key_bias, s),
                                                            _block_mask_ptr(block_mask, s), s._call.ref, scale,
                                                            _q(O, s), ws.data_ptr(), ws.numel() * ws.element_size(),
                                                            _stream())
    _check("dense_attention_fused_blocked_split", st)
    return O


def dfss_spmm_t(vals, meta, X, s: Shape, out=None):
    """Transposed sparse product A^T X -> bf16 [BH, Lk, d] (dV = P^T dO, dK = dS^T Q)."""
    if out is None:
        out = torch.empty((s.BH, s.Lk, s.d), dtype=s.torch_dtype, device=X.device)
    st = load_library().dfss_spmm_t(_kept(vals, s), _meta(meta, s), _q(X, s),
                                    s._call.ref, _kv(out, s), _stream())
    _check("dfss_spmm_t", st)
    return out


def dfss_backward_workspace_bytes(s: Shape) -> int:
    return int(load_library().dfss_backward_workspace_bytes(s._call.ref))


def dfss_attention_backward(dO, Q, K, V, O, P, meta, s: Shape, scale: float, dQ=None, dK=None, dV=None, ws=None):
    """Gradients through the fixed selection.  P, meta: weights and metadata kept from the forward stages."""
    if dQ is None:
        dQ = torch.empty(s._call.O_shape, dtype=s._call.torch_dtype, device=Q.device)
    if dK is None:
        dK = torch.empty((s.BH, s.Lk, s.d), dtype=s.torch_dtype, device=Q.device)
    if dV is None:
        dV = torch.empty((s.BH, s.Lk, s.d), dtype=s.torch_dtype, device=Q.device)
    if ws is None:
        ws = _alloc_bytes(dfss_backward_workspace_bytes(s), Q.device)
    st = load_library().dfss_attention_backward(_q(dO, s), _q(Q, s), _kv(K, s), _kv(V, s), _q(O, s),
                                                _kept(P, s), _meta(meta, s), s._call.ref, scale,
                                                _q(dQ, s), _kv(dK, s),
                                                _kv(dV, s), _ptr(ws),
                                                ws.numel() * ws.element_size(), _stream())
    _check("dfss_attention_backward", st)
    return dQ, dK, dV


def dfss_meta_to_canonical(meta, s: Shape, canon=None):
    """Library word order -> canonical uint16 [BH, Lq, Lk/16] (held as int16 bits)."""
    if canon is None:
        canon = torch.empty((s.BH, s.LqP, s.meta_words), dtype=torch.int16, device=meta.device)
    st = load_library().dfss_meta_to_canonical(_meta(meta, s), s._call.ref, _meta(canon, s), _stream())
    _check("dfss_meta_to_canonical", st)
    return canon


def dfss_meta_from_canonical(canon, s: Shape, meta=None):
    if meta is None:
        meta = torch.empty((s.BH * s.LqP * s.meta_words,), dtype=torch.int16, device=canon.device)
    st = load_library().dfss_meta_from_canonical(_meta(canon, s), s._call.ref, _meta(meta, s), _stream())
    _check("dfss_meta_from_canonical", st)
    return meta


def internal_plan(call: str, *sizes: int):
    """Which instances a decoder's call ("norm", "append", "cached") runs (tests only; csrc/dfss_internal.h): whole numbers."""
    out = (ctypes.c_int32 * (4 if call == "cached" else 3))()
    f = getattr(load_library(), f"dfss_internal_{call}_plan")
    f.restype = None
    f(*(ctypes.c_int32(x) for x in sizes), out)
    return tuple(out)


# ---- around a decoder's attention ------------------------------------------------------------------------------


def _current(device: int) -> bool:
    """Whether that is the current device (-1: the host's)."""
    return device >= 0 and device == torch._C._cuda_getDevice()


def _array(t: torch.Tensor, dtype, shape, device: int | None, what: str) -> int:
    """Pointer of a contiguous tensor of the given type (or of one of several) and shape, on the current device, or on the
    given one, which is known to be that."""
    there = t.get_device()
    if t.dtype is dtype and t.shape == shape and (there == device or device is None and _current(there)) and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype and not (isinstance(dtype, tuple) and t.dtype in dtype):
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor {list(shape)}, got {list(t.shape)}")
    if not _current(there):
        raise ValueError(f"{what}: expected a tensor on the current device, got one on {t.device}")
    return t.data_ptr()


def _read_only(slot: str) -> property:
    """What an object was made of, to be read: the pointers that its calls pass on were taken then."""
    return property(attrgetter(slot))


class Rotary:
    """Rotary positions (``dfss_rotary``): cos, sin float32 [n_pos, rot/2]; pos int32, the position of every token of a
    call (None: its place in its sequence); pairs (i, i + rot/2), or neighbours if ``interleaved``.  Keeps its tensors, which
    cannot be exchanged for others (their contents can): another tensor is another Rotary."""
    __slots__ = ("_cos", "_sin", "_pos", "_interleaved", "_device", "_c")
    cos, sin, pos, interleaved, device = map(_read_only, __slots__[:5])

    def __init__(self, cos, sin, pos=None, interleaved: bool = False):
        shape, f = cos.shape, torch.float32
        if len(shape) != 2:
            raise ValueError(f"cos, sin: expected [n_pos, rot/2], got {list(shape)}")
        self._cos, self._sin, self._pos, self._interleaved = cos, sin, pos, interleaved
        self._device = dev = cos.get_device()
        if not (_current(dev) and cos.dtype is f and sin.dtype is f and sin.shape == shape and sin.get_device() == dev
                and cos.is_contiguous() and sin.is_contiguous()):
            _array(cos, f, shape, None, "cos"), _array(sin, f, shape, dev, "sin")   # says what is wrong
        self._c = _ROTARY.pack(cos.data_ptr(), sin.data_ptr(), 0 if pos is None else _array(pos, torch.int32, pos.shape, dev, "pos"),
                               shape[0], 2 * shape[1], 1 if interleaved else 0)


def _rotary(r: Rotary | None, tokens: int):
    if r is None:
        return None
    if r._pos is not None and r._pos.numel() != tokens:
        raise ValueError(f"pos: expected {tokens} positions, got {r._pos.numel()}")
    if not _current(r._device):
        raise ValueError(f"rotary: expected one on the current device, got one on {r.cos.device}")
    return r._c


_CODES = (torch.uint8, torch.float8_e4m3fn)


class Cache:
    """A paged cache of 8 bits (``dfss_cache``): k, v uint8 or float8_e4m3fn [n_pages, Hk, page, d], their scales float32
    [n_pages, Hk], table int32 [B, width], len int32 [B].  Keeps its tensors, which cannot be exchanged for others (their contents
    can): another table, say, is another Cache."""
    __slots__ = ("_k", "_v", "_k_scale", "_v_scale", "_table", "_len", "_B", "_Hk", "_d", "_device", "_c")
    k, v, k_scale, v_scale, table, len, B, Hk, d, device = map(_read_only, __slots__[:10])

    def __init__(self, k, v, k_scale, v_scale, table, len):
        shape, where, f, i = k.shape, table.shape, torch.float32, torch.int32
        if k.dim() != 4 or table.dim() != 2:
            raise ValueError(f"expected k, v [n_pages, Hk, page, d] and table [B, width], got {list(shape)}, {list(where)}")
        self._k, self._v, self._k_scale, self._v_scale, self._table, self._len = k, v, k_scale, v_scale, table, len
        n, Hk, page, self._d = shape
        B, width = where
        self._Hk, self._B = Hk, B
        scales, codes, lens = (n, Hk), k.dtype, (B,)
        self._device = dev = k.get_device()
        if not (codes in _CODES and v.dtype is codes and k_scale.dtype is f and v_scale.dtype is f and table.dtype is i and len.dtype is i
                and v.shape == shape and k_scale.shape == scales and v_scale.shape == scales and len.shape == lens
                and _current(dev) and v.get_device() == dev and k_scale.get_device() == dev and v_scale.get_device() == dev
                and table.get_device() == dev and len.get_device() == dev and k.is_contiguous() and v.is_contiguous()
                and k_scale.is_contiguous() and v_scale.is_contiguous() and table.is_contiguous() and len.is_contiguous()):
            # says what is wrong
            _array(k, codes if codes in _CODES else _CODES, shape, None, "k"), _array(v, codes, shape, dev, "v")
            _array(k_scale, f, scales, dev, "k_scale"), _array(v_scale, f, scales, dev, "v_scale")
            _array(table, i, where, dev, "table"), _array(len, i, lens, dev, "len")
        self._c = _CACHE.pack(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), table.data_ptr(), len.data_ptr(),
                              n, Hk, page, width)


def _scratch(ws: torch.Tensor | None) -> int | None:
    """Pointer of a workspace of the caller's."""
    p = _ptr(ws)
    if ws is not None and not _current(ws.get_device()):
        raise ValueError(f"ws: expected a tensor on the current device, got one on {ws.device}")
    return p


def _rows(t: torch.Tensor | None, shape, dtype, what: str, out: bool = False):
    """Rows of heads, as bytes, and their number of heads (None, 0 without a tensor): [batch, token, head, d] with any strides of the first
    three, or the contiguous [batch * head, token, d] of the attention calls, for a shape (batch, token, d); [token, head, d]
    with any strides of the first two for a shape (token, d)."""
    if t is None:
        return None, 0
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    n, x, d, dims = t.shape, t.stride(), shape[-1], t.dim()
    if len(shape) == 2:
        if dims != 3 or n[0] != shape[0] or n[2] != d or x[2] != 1:
            raise ValueError(f"{what}: expected [{shape[0]}, heads, {d}] with elements side by side, got {list(n)}")
        H, batch, token, head = n[1], 0, x[0] if n[0] > 1 else 0, x[1] if n[1] > 1 else 0
    elif dims == 3:
        if shape[0] < 1 or n[0] % shape[0] or n[1] != shape[1] or n[2] != d or not t.is_contiguous():
            raise ValueError(f"{what}: expected a contiguous [{shape[0]} * heads, {shape[1]}, {d}], got {list(n)}")
        H = n[0] // shape[0]
        batch, token, head = H * shape[1] * d, d, shape[1] * d
    else:
        if dims != 4 or n[0] != shape[0] or n[1] != shape[1] or n[3] != d or x[3] != 1:
            raise ValueError(f"{what}: expected [{shape[0]}, {shape[1]}, heads, {d}] with elements side by side, got {list(n)}")
        H, batch, token, head = n[2], x[0] if n[0] > 1 else 0, x[1] if n[1] > 1 else 0, x[2] if n[2] > 1 else 0
    if out and 0 in x and any(k > 1 and y == 0 for k, y in zip(n, x)):
        raise ValueError(f"{what}: a result cannot share rows")
    if not _current(t.get_device()):
        raise ValueError(f"{what}: expected a tensor on the current device, got one on {t.device}")
    return _ROWS.pack(t.data_ptr(), H, batch, token, head), H


def _headed(X: torch.Tensor, B: int, H: int, L: int, d: int):
    """A new [B * H, L, d] of X's type and device, and its rows, as _rows gives them."""
    t = X.new_empty((B * H, L, d))
    return t, _ROWS.pack(t.data_ptr(), H, H * L * d, d, L * d)


def _weight(w: torch.Tensor | None, dtype, d: int, what: str):
    return None if w is None else _array(w, dtype, (d,), None, what)


def dfss_qk_norm_rotate(Q, K, wq, wk, rotary: Rotary | None, s: Shape, eps: float = 1e-6, Qo=None, Ko=None):
    """Norm of every head's query and key (weights wq, wk [d], None: none) and rotation to the token's position.
    Q, K: [B, Lq, heads, d] with any strides (or [B * heads, Lq, d]); K may be None.  Returns Qo, Ko, [B * heads, Lq, d] as
    the attention calls take them unless given."""
    t, shape = s._call.torch_dtype, (s.B, s.Lq, s.d)
    (q, Hq), (k, Hk) = _rows(Q, shape, t, "Q"), _rows(K, shape, t, "K")
    if Qo is None:
        Qo, qo = _headed(Q, s.B, Hq, s.Lq, s.d)
    else:
        qo = _rows(Qo, shape, t, "Qo", True)[0]
    if Ko is None and K is not None:
        Ko, ko = _headed(K, s.B, Hk, s.Lq, s.d)
    else:
        ko = _rows(Ko, shape, t, "Ko", True)[0]
    st = load_library().dfss_qk_norm_rotate(q, k, _weight(wq, t, s.d, "wq"), _weight(wk, t, s.d, "wk"),
                                            _rotary(rotary, s.B * s.Lq), s._call.ref, eps, qo, ko, _stream())
    _check("dfss_qk_norm_rotate", st)
    return Qo, Ko


def dfss_qk_norm_workspace_bytes(s: Shape) -> int:
    return int(load_library().dfss_qk_norm_workspace_bytes(s._call.ref))


def dfss_qk_norm_rotate_backward(dQo, dKo, Q, K, wq, wk, rotary: Rotary | None, s: Shape, eps: float = 1e-6, dQ=None, dK=None,
                                 dwq=None, dwk=None, ws=None):
    """Gradients of dfss_qk_norm_rotate: (dQ, dK, dwq, dwk), those of Q and K [B, Lq, heads, d] unless given, those of the
    weights float32 [d] (None where there is no weight)."""
    t, shape = s._call.torch_dtype, (s.B, s.Lq, s.d)
    (q, Hq), (k, Hk) = _rows(Q, shape, t, "Q"), _rows(K, shape, t, "K")
    if dQ is None:
        dQ = Q.new_empty((s.B, s.Lq, Hq, s.d))
    if dK is None and K is not None:
        dK = K.new_empty((s.B, s.Lq, Hk, s.d))
    if dwq is None and wq is not None:
        dwq = torch.empty(s.d, dtype=torch.float32, device=Q.device)
    if dwk is None and wk is not None and K is not None:
        dwk = torch.empty(s.d, dtype=torch.float32, device=Q.device)
    if ws is None and (dwq is not None or dwk is not None):
        ws = _alloc_bytes(dfss_qk_norm_workspace_bytes(s), Q.device)
    st = load_library().dfss_qk_norm_rotate_backward(
        _rows(dQo, shape, t, "dQo")[0], _rows(dKo, shape, t, "dKo")[0], q, k, _weight(wq, t, s.d, "wq"), _weight(wk, t, s.d, "wk"),
        _rotary(rotary, s.B * s.Lq), s._call.ref, eps, _rows(dQ, shape, t, "dQ", True)[0], _rows(dK, shape, t, "dK", True)[0],
        _weight(dwq, torch.float32, s.d, "dwq"), _weight(dwk, torch.float32, s.d, "dwk"), _scratch(ws),
        0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check("dfss_qk_norm_rotate_backward", st)
    return dQ, dK, dwq, dwk


def _offsets(cu: torch.Tensor | None, s: Shape):
    return None if cu is None else _array(cu, torch.int32, (s.B + 1,), None, "cu")


def _cache(c: Cache, s: Shape):
    if c._B != s.B or c._d != s.d:
        raise ValueError(f"cache: expected {s.B} sequences and head size {s.d}, got {c._B} and {c._d}")
    if not _current(c._device):
        raise ValueError(f"cache: expected one on the current device, got one on {c._k.device}")
    return c._c


def dfss_cache_append(K, V, cu, cache: Cache, w, rotary: Rotary | None, s: Shape, eps: float = 1e-6):
    """New tokens into the cache: K, V [tokens, Hk, d] with any strides of the first two, tokens cu[b] .. cu[b+1] - 1 for
    sequence b (cu None: Lq each); cache.len holds the lengths with them.  Keys are normed (w None: not) and rotated on
    the way.  s: B sequences, H = Hk key heads, at most Lk tokens a sequence."""
    n = K.shape[0]
    st = load_library().dfss_cache_append(_rows(K, (n, s.d), torch.bfloat16, "K")[0], _rows(V, (n, s.d), torch.bfloat16, "V")[0], n,
                                          _offsets(cu, s), _cache(cache, s), _weight(w, torch.bfloat16, s.d, "w"),
                                          _rotary(rotary, n), s._call.ref, eps, _stream())
    _check("dfss_cache_append", st)


def dfss_cached_workspace_bytes(s: Shape, cache: Cache) -> int:
    return int(load_library().dfss_cached_workspace_bytes(s._call.ref, cache._c))


def _attention_cached(name: str, Q, cu, cache: Cache, s: Shape, scale: float, causal: bool, O, ws):
    n = Q.shape[0]
    (q, H), c = _rows(Q, (n, s.d), torch.bfloat16, "Q"), _cache(cache, s)
    if O is None:
        O = Q.new_empty((n, H, s.d))
        o = O.data_ptr()
    else:
        o = _array(O, torch.bfloat16, (n, H, s.d), None, "O")
    L = load_library()
    w = None
    if ws is not None:
        need, w = ws.numel() * ws.element_size(), _scratch(ws)
    else:
        need = s._call.cached_ws.get(cache._Hk)      # (of a valid shape it depends on nothing else of the cache)
        if not need:
            need = s._call.cached_ws[cache._Hk] = L.dfss_cached_workspace_bytes(s._call.ref, c)
        if need:
            ws = _alloc_bytes(need, Q.device)
            w = ws.data_ptr()
    st = getattr(L, name)(q, n, None if cu is None else _array(cu, torch.int32, (s.B + 1,), None, "cu"), c, s._call.ref, scale,
                          1 if causal else 0, o, w, need, _stream())
    _check(name, st)
    return O


def dfss_attention_cached(Q, cu, cache: Cache, s: Shape, scale: float, causal: bool = True, O=None, ws=None):
    """N:M pruned attention of queries [tokens, H, d] (any strides of the first two; offsets cu as in dfss_cache_append) over
    the cache; causal: they are the last tokens of their sequences.  s: B sequences, H query heads, at most Lq queries and
    Lk keys a sequence, N of M.  Returns O [tokens, H, d]."""
    return _attention_cached("dfss_attention_cached", Q, cu, cache, s, scale, causal, O, ws)


def dense_attention_cached(Q, cu, cache: Cache, s: Shape, scale: float, causal: bool = True, O=None, ws=None):
    """Full attention over the cache; arguments as dfss_attention_cached (N, M ignored)."""
    return _attention_cached("dense_attention_cached", Q, cu, cache, s, scale, causal, O, ws)
