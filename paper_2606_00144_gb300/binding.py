"""Thin ctypes binding of libbudgetdraft (include/budgetdraft.h).

Argument marshalling only: every computation runs in the library's CUDA kernels.  torch
tensors provide device memory and the current CUDA stream.  There is no fallback: if
the library is not built, or an argument is rejected, these functions raise.
"""

from __future__ import annotations

import ctypes
import functools
import math
import os
import struct

import torch

from .build import LIB_PATH

BD_OK = 0
BD_ERR_CUDA = -5
BD_OP_SELECT, BD_OP_DRAFT, BD_OP_VERIFY, BD_OP_QUANT_DRAFT, BD_OP_QUANT_VERIFY = 1, 2, 3, 4, 5
BD_OP_PAGED_DRAFT, BD_OP_PAGED_VERIFY = 6, 7
BD_PAGED_BLOCK_ROWS = -1
BD_QUANT_BLOCK_ROWS = -1
BD_QUANT_GROUP = 32
BD_DRAFT_VIEW_READY = 1
BD_SELECT_WINDOW_READY, BD_SELECT_NAN_HIDDEN = 1, 4
BD_DTYPE_BF16, BD_DTYPE_F32 = 1, 2


class BdShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("t_ctx", ctypes.c_int32), ("t_cap", ctypes.c_int32),
                ("seq_lens", ctypes.c_void_p)]

    def __repr__(self):
        return (f"BdShape(batch={self.batch}, h_q={self.h_q}, h_kv={self.h_kv}, head_dim={self.head_dim}, "
                f"t_ctx={self.t_ctx}, t_cap={self.t_cap})")


class BdQuantCache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p)]


class BdPagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_strides", ctypes.c_int64 * 3),
                ("v_strides", ctypes.c_int64 * 3), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class BdRope(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class BudgetDraftError(RuntimeError):
    def __init__(self, func, status):
        self.status = status
        super().__init__(f"{func} failed: {bd_strerror(status)} ({status})")


_lib = None
_P = ctypes.c_void_p
_SHAPE = ctypes.POINTER(BdShape)
_QCACHE = ctypes.POINTER(BdQuantCache)
_STRIDES = ctypes.POINTER(ctypes.c_int64)
_PCACHE = ctypes.POINTER(BdPagedCache)
_ROPE = ctypes.POINTER(BdRope)
_SIGNATURES = {
    "bd_workspace_size": (ctypes.c_size_t, [_SHAPE, ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "bd_select_budget": (ctypes.c_int, [_SHAPE, _P, _P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                        ctypes.c_int, ctypes.c_int, ctypes.c_uint, _P, _P, _P, ctypes.c_size_t,
                                        _P]),
    "bd_draft_attn": (ctypes.c_int, [_SHAPE, _P, _P, _P, _P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_uint, _P,
                                     _P, _P, ctypes.c_size_t, _P]),
    "bd_draft_attn_static": (ctypes.c_int, [_SHAPE, _P, _P, _P, _P, _P, ctypes.c_int, ctypes.c_int, _P, _P,
                                            _P]),
    "bd_draft_static_status": (ctypes.c_int, [_P]),
    "bd_verify_attn": (ctypes.c_int, [_SHAPE, _P, ctypes.c_int, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "bd_combine": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_int, _P, _P, _P]),
    "bd_argmax": (ctypes.c_int, [_P, ctypes.c_int, ctypes.c_int, ctypes.c_int, _P, _P]),
    "bd_accept": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P]),
    "bd_advance": (ctypes.c_int, [_SHAPE, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, ctypes.c_int, _P,
                                  _P]),
    "bd_write_block_rows": (ctypes.c_int, [_SHAPE, ctypes.c_int, _P, _P, _P, _P, _P]),
    "bd_quant_write": (ctypes.c_int, [_SHAPE, ctypes.c_int, ctypes.c_int, _P, _STRIDES, _P, _STRIDES, _QCACHE, _P]),
    "bd_quant_read": (ctypes.c_int, [_SHAPE, ctypes.c_int, ctypes.c_int, ctypes.c_int, _QCACHE, _P, _STRIDES, _P,
                                     _STRIDES, _P]),
    "bd_quant_draft_attn": (ctypes.c_int, [_SHAPE, _P, _QCACHE, _P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_uint, _P,
                                           _P, _P, ctypes.c_size_t, _P]),
    "bd_quant_verify_attn": (ctypes.c_int, [_SHAPE, _P, ctypes.c_int, _QCACHE, _P, _P, _P, ctypes.c_size_t, _P]),
    # (strides as packed bytes: an array of them takes a call 0.2 us more to make and to pass)
    "bd_paged_append": (ctypes.c_int, [_SHAPE, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P,
                                       _ROPE, _PCACHE, _P, ctypes.c_int, _P, _P, _P]),
    "bd_paged_read": (ctypes.c_int, [_SHAPE, ctypes.c_int, ctypes.c_int, _PCACHE, _P, ctypes.c_int, _P, _P, _P,
                                     _P, _P]),
    "bd_paged_keys": (ctypes.c_int, [_SHAPE, ctypes.c_int, _PCACHE, _P, ctypes.c_int, _P, _P, _P]),
    "bd_paged_verify_attn": (ctypes.c_int, [_SHAPE, _P, ctypes.c_int, _PCACHE, _P, ctypes.c_int, _P, _P, _P,
                                            ctypes.c_size_t, _P]),
    "bd_paged_draft_attn": (ctypes.c_int, [_SHAPE, _P, _PCACHE, _P, ctypes.c_int, _P, _P, ctypes.c_int, ctypes.c_int,
                                           ctypes.c_uint, _P, _P, _P, ctypes.c_size_t, _P]),
    "bd_check_wait_timeout": (ctypes.c_int, [_P, ctypes.c_size_t, ctypes.c_int, _P]),
    "bd_workspace_status": (ctypes.c_int, [_P, _P]),
    "bd_strerror": (ctypes.c_char_p, [ctypes.c_int]),
}


def library():
    """Load libbudgetdraft.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run paper_2606_00144_gb300.build.build() first")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def exported_symbols():
    return list(_SIGNATURES)


def bd_strerror(status: int) -> str:
    return library().bd_strerror(int(status)).decode()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # the handle alone: building the Stream object takes 3 us of a call's 9
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(name, status):
    if status != BD_OK:
        raise BudgetDraftError(name, status)


def make_shape(batch, h_q, h_kv, head_dim, t_ctx, t_cap, seq_lens=None) -> BdShape:
    """seq_lens: optional int32 device tensor [batch] of per-sequence context lengths (t_ctx
    is then the longest); the tensor must outlive every call made with this shape."""
    return BdShape(int(batch), int(h_q), int(h_kv), int(head_dim), int(t_ctx), int(t_cap), _ptr(seq_lens))


def shape_of(k_cache: torch.Tensor, h_q: int, t_ctx: int) -> BdShape:
    b, h_kv, t_cap, d = k_cache.shape
    return make_shape(b, h_q, h_kv, d, t_ctx, t_cap)


def bd_workspace_size(shape: BdShape, op: int, budget: int, n_q: int) -> int:
    return int(library().bd_workspace_size(ctypes.byref(shape), op, int(budget), int(n_q)))


class Workspace:
    """A device buffer sized for a set of operations (see bd_workspace_size), zero-filled: as a
    whole, or with ``units`` (batch * h_kv) given only the status word and the arrival counters, the
    part that the kernels read before they write it."""

    def __init__(self, nbytes: int, device=None, units: int | None = None):
        self.nbytes = int(max(nbytes, 512))
        if units is None:
            self.buf = torch.zeros(self.nbytes, dtype=torch.uint8, device=device or "cuda")
        else:
            self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device or "cuda")
            self.buf[:256 + -(-4 * units // 256) * 256].zero_()

    @classmethod
    def for_step(cls, shape: BdShape, budget: int, window: int, gamma: int, device=None):
        sizes = [bd_workspace_size(shape, BD_OP_SELECT, budget, window),
                 bd_workspace_size(shape, BD_OP_DRAFT, budget, gamma),
                 bd_workspace_size(shape, BD_OP_VERIFY, budget, gamma + 1)]
        # an op this shape does not support reports size 0 here and its status when called
        if max(sizes) == 0:
            raise BudgetDraftError("bd_workspace_size", -1)
        return cls(max(sizes), device)

    @property
    def ptr(self):
        return self.buf.data_ptr()

    def status(self, stream=None) -> int:
        return int(library().bd_workspace_status(self.ptr, _stream(stream)))


def bd_select_budget(shape, k_cache, q_window, window_lse, window, budget, n_sink, n_recent, chunk,
                     idx_out, count_out, ws: Workspace, stream=None, flags=0):
    st = library().bd_select_budget(ctypes.byref(shape), _ptr(k_cache), _ptr(q_window), _ptr(window_lse),
                                    int(window), int(budget), int(n_sink), int(n_recent), int(chunk),
                                    int(flags), _ptr(idx_out), _ptr(count_out), ws.ptr, ws.nbytes,
                                    _stream(stream))
    _check("bd_select_budget", st)


def bd_draft_attn(shape, q, k_cache, v_cache, idx, count, budget, step_j, o_out, lse_out,
                  ws: Workspace, stream=None, flags=0):
    st = library().bd_draft_attn(ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(idx),
                                 _ptr(count), int(budget), int(step_j), int(flags), _ptr(o_out), _ptr(lse_out),
                                 ws.ptr, ws.nbytes, _stream(stream))
    _check("bd_draft_attn", st)


def bd_draft_attn_static(shape, q, k_cache, v_cache, idx, count, budget, step_j, o_out, lse_out, stream=None):
    """bd_draft_attn for callers that cannot allocate device memory: no workspace; the
    library's own 4 MiB device array holds the scratch, shared by every call (calls must
    not overlap on the GPU; the first call on a device must precede any stream capture)."""
    st = library().bd_draft_attn_static(ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(idx),
                                        _ptr(count), int(budget), int(step_j), _ptr(o_out), _ptr(lse_out),
                                        _stream(stream))
    _check("bd_draft_attn_static", st)


def bd_draft_static_status(stream=None) -> int:
    """Reads and clears the device-side error word of bd_draft_attn_static's array."""
    st = library().bd_draft_static_status(_stream(stream))
    if st == BD_ERR_CUDA:
        _check("bd_draft_static_status", st)
    return int(st)


def bd_verify_attn(shape, q, n_q, k_cache, v_cache, o_out, lse_out, ws: Workspace, stream=None):
    st = library().bd_verify_attn(ctypes.byref(shape), _ptr(q), int(n_q), _ptr(k_cache), _ptr(v_cache),
                                  _ptr(o_out), _ptr(lse_out), ws.ptr, ws.nbytes, _stream(stream))
    _check("bd_verify_attn", st)


def bd_combine(o_part, lse_part, n_split, rows, head_dim, o_out, lse_out, stream=None):
    st = library().bd_combine(_ptr(o_part), _ptr(lse_part), int(n_split), int(rows), int(head_dim),
                              _ptr(o_out), _ptr(lse_out), _stream(stream))
    _check("bd_combine", st)


def bd_argmax(logits, ids_out, stream=None):
    """ids_out[r] = arg max of logits[r] (bf16 or fp32 [rows, vocab], int32 [rows])."""
    if logits.dtype == torch.bfloat16:
        dtype = BD_DTYPE_BF16
    elif logits.dtype == torch.float32:
        dtype = BD_DTYPE_F32
    else:
        raise TypeError(f"bd_argmax: logits must be bf16 or fp32, got {logits.dtype}")
    if logits.dim() != 2 or not logits.is_contiguous():
        raise ValueError("bd_argmax: logits must be a contiguous [rows, vocab] tensor")
    rows, vocab = logits.shape
    st = library().bd_argmax(_ptr(logits), dtype, int(rows), int(vocab), _ptr(ids_out), _stream(stream))
    _check("bd_argmax", st)


def bd_accept(draft_tokens, verify_tokens, n_accept_out, emit_out, stream=None):
    """Accepted prefix length and emitted tokens: draft_tokens int32 [gamma, batch] (pass-major),
    verify_tokens int32 [batch, gamma + 1]."""
    batch, g1 = verify_tokens.shape
    st = library().bd_accept(int(batch), int(g1 - 1), _ptr(draft_tokens), _ptr(verify_tokens), _ptr(n_accept_out),
                             _ptr(emit_out), _stream(stream))
    _check("bd_accept", st)


def bd_advance(shape, window, n_q, n_accept, q_verify, verify_lse, q_window, window_lse, idx=None, count=None,
               advance_out=None, stream=None):
    """Slides the observation window (and appends to the sparse view) after acceptance."""
    cap = int(idx.shape[-1]) if idx is not None else 0
    st = library().bd_advance(ctypes.byref(shape), int(window), int(n_q), _ptr(n_accept), _ptr(q_verify),
                              _ptr(verify_lse), _ptr(q_window), _ptr(window_lse), _ptr(idx), _ptr(count), cap,
                              _ptr(advance_out), _stream(stream))
    _check("bd_advance", st)


def bd_write_block_rows(shape, n_rows, k_rows, v_rows, k_cache, v_cache, stream=None):
    """Writes rows t_ctx .. t_ctx + n_rows - 1 of the caches from dense [b, h_kv, n_rows, d]
    buffers (device or pinned host memory)."""
    st = library().bd_write_block_rows(ctypes.byref(shape), int(n_rows), _ptr(k_rows), _ptr(v_rows), _ptr(k_cache),
                                       _ptr(v_cache), _stream(stream))
    _check("bd_write_block_rows", st)


class QuantCache:
    """A 4-bit KV cache (the format is in the header): uint8 codes [batch, h_kv, t_cap, head_dim / 2]
    and bf16 scales [batch, h_kv, t_cap, head_dim / 32] of K and of V.  The tensors stay the caller's:
    they may be views that other code reads, as long as each is dense."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        if k_codes.dim() != 4 or k_codes.shape[3] not in (32, 64):
            raise ValueError("QuantCache: codes must be [batch, h_kv, t_cap, head_dim / 2] with head_dim 64 or 128")
        self.batch, self.h_kv, self.t_cap = (int(x) for x in k_codes.shape[:3])
        self.head_dim = 2 * int(k_codes.shape[3])
        for codes, scales in ((k_codes, k_scales), (v_codes, v_scales)):
            if codes.dtype != torch.uint8 or scales.dtype != torch.bfloat16:
                raise TypeError("QuantCache: codes are uint8, scales bf16")
            if codes.shape != k_codes.shape or tuple(scales.shape) != (*k_codes.shape[:3], self.head_dim // BD_QUANT_GROUP):
                raise ValueError("QuantCache: codes and scales must cover the same rows")
            if not (codes.is_contiguous() and scales.is_contiguous()):
                raise ValueError("QuantCache: codes and scales must be contiguous")
            if codes.device != k_codes.device or scales.device != k_codes.device:
                raise ValueError("QuantCache: codes and scales must be on one device")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self._rows = (self.batch, self.h_kv, self.head_dim, self.t_cap)
        self._struct = BdQuantCache(_ptr(k_codes), _ptr(k_scales), _ptr(v_codes), _ptr(v_scales))
        self._ref = ctypes.byref(self._struct)
        self.is_cuda = k_codes.is_cuda
        self._gpu = k_codes.get_device() if self.is_cuda else None   # (what no tensor's get_device() equals where it is none)

    @classmethod
    def empty(cls, batch, h_kv, t_cap, head_dim, device="cuda"):
        """A cache whose rows are not written yet."""
        def one():
            return (torch.empty(batch, h_kv, t_cap, head_dim // 2, dtype=torch.uint8, device=device),
                    torch.empty(batch, h_kv, t_cap, head_dim // BD_QUANT_GROUP, dtype=torch.bfloat16, device=device))
        return cls(*one(), *one())

    def shape(self, h_q: int, t_ctx: int, seq_lens=None) -> BdShape:
        return make_shape(self.batch, h_q, self.h_kv, self.head_dim, t_ctx, self.t_cap, seq_lens)

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k_codes, self.k_scales, self.v_codes, self.v_scales))


# The calls below are small next to a launch, so what they check is checked once, in one place, and told apart
# (_refuse_rows, _refuse) only when something does not fit.
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32
_shape_ints = struct.Struct("6i").unpack_from      # a shape's sizes at once


@functools.lru_cache(maxsize=256)
def _stride_array(sb, sh, sn):
    return (ctypes.c_int64 * 3)(sb, sh, sn)


def _refuse_cache(name, shape):
    raise ValueError(f"{name}: the cache is not one of this shape: {shape}")


def _refuse_rows(name, want, dtype, *rows):
    for t in (x for x in rows if x is not None):
        if t.shape != want:
            raise ValueError(f"{name}: rows must be [batch, h_kv, n, head_dim] = {want}, got {tuple(t.shape)}")
        if t.dtype is not dtype or dtype not in (_BF16, _F32):
            raise TypeError(f"{name}: rows must be bf16 or fp32, K and V alike, got {t.dtype}")
        if not t.is_contiguous() and t.stride(3) != 1:
            raise ValueError(f"{name}: the elements of a row must be adjacent")
    raise ValueError(f"{name}: the rows and the cache must be on the GPU, the same one")


def _quant_rows(name, shape, cache, k_rows, v_rows):
    """Checks a write's or read's cache and tensors [batch, h_kv, n, head_dim]: n, the dtype's code, the tensors'
    pointers and strides (None where they are dense)."""
    first = k_rows if k_rows is not None else v_rows
    if first is None:
        raise ValueError(f"{name}: K rows, V rows or both")
    b, _, h, d, _, cap = _shape_ints(shape)
    if (b, h, d, cap) != cache._rows:
        _refuse_cache(name, shape)
    dtype = first.dtype
    want = (b, h, first.shape[2] if first.dim() == 4 else -1, d)
    out, gpu = [], cache._gpu
    for t in (k_rows, v_rows):
        if t is None:
            out += None, None
            continue
        if not (t.shape == want and t.dtype is dtype and (dtype is _BF16 or dtype is _F32) and t.get_device() == gpu):
            _refuse_rows(name, want, dtype, k_rows, v_rows)
        if t.is_contiguous():
            out += t.data_ptr(), None
            continue
        sb, sh, sn, one = t.stride()
        if one != 1:
            _refuse_rows(name, want, dtype, k_rows, v_rows)
        out += t.data_ptr(), _stride_array(sb, sh, sn)
    return want[2], BD_DTYPE_BF16 if dtype is _BF16 else BD_DTYPE_F32, out


def _refuse(name, **tensors):
    for what, (t, dtype, shape) in tensors.items():
        if t is not None and t.dtype is not dtype:
            raise TypeError(f"{name}: {what} must be {dtype}, got {t.dtype}")
        if t is not None and (t.shape != shape or not t.is_contiguous()):
            raise ValueError(f"{name}: {what} must be a contiguous {shape} tensor, got {tuple(t.shape)}")
    raise ValueError(f"{name}: every tensor must be on the GPU of the cache")


def _quant_attn(name, shape, cache, q, o_out, lse_out, n_q, idx=None, count=None, budget=0):
    """Checks the cache, the queries (of a drafter pass where n_q is None), the outputs and a drafter pass's view."""
    b, h_q, h, d, _, cap = _shape_ints(shape)
    if (b, h, d, cap) != cache._rows:
        _refuse_cache(name, shape)
    want = (b, h_q, d) if n_q is None else (b, h_q, n_q, d)
    units, gpu = (b, h), cache._gpu
    if not (q.dtype is _BF16 and o_out.dtype is _BF16 and q.shape == want and o_out.shape == want and q.is_contiguous()
            and o_out.is_contiguous() and q.get_device() == gpu and o_out.get_device() == gpu
            and (lse_out is None or (lse_out.dtype is _F32 and lse_out.shape == want[:-1] and lse_out.is_contiguous()
                                     and lse_out.get_device() == gpu))
            and (idx is None or (idx.dtype is _I32 and count.dtype is _I32 and idx.shape == (b, h, budget)
                                 and count.shape == units and idx.is_contiguous() and count.is_contiguous()
                                 and idx.get_device() == gpu and count.get_device() == gpu))):
        _refuse(name, q=(q, _BF16, want), o_out=(o_out, _BF16, want), lse_out=(lse_out, _F32, want[:-1]),
                idx=(idx, _I32, (*units, budget)), count=(count, _I32, units))


def bd_quant_write(shape, k_rows, v_rows, cache: QuantCache, stream=None):
    """Quantises rows [batch, h_kv, n, head_dim] (bf16 or fp32; any strides of whole 16 bytes; either may
    be None) into the cache, behind the context (each sequence's length, if the shape has lengths)."""
    n, dtype, (k, ks, v, vs) = _quant_rows("bd_quant_write", shape, cache, k_rows, v_rows)
    st = (_lib or library()).bd_quant_write(ctypes.byref(shape), n, dtype, k, ks, v, vs, cache._ref, _stream(stream))
    _check("bd_quant_write", st)


def bd_quant_read(shape, cache: QuantCache, k_out, v_out=None, first_row=None, stream=None):
    """Reads the cache's rows first_row .. first_row + n - 1 (None: those behind the context) into
    [batch, h_kv, n, head_dim] tensors, bf16 or fp32; either may be None."""
    n, dtype, (k, ks, v, vs) = _quant_rows("bd_quant_read", shape, cache, k_out, v_out)
    if first_row is None:
        first_row = BD_QUANT_BLOCK_ROWS
    elif first_row < 0:
        raise ValueError("bd_quant_read: first_row must not be negative")
    st = (_lib or library()).bd_quant_read(ctypes.byref(shape), first_row, n, dtype, cache._ref, k, ks, v, vs, _stream(stream))
    _check("bd_quant_read", st)


def bd_quant_draft_attn(shape, q, cache: QuantCache, idx, count, budget, step_j, o_out, lse_out, ws: Workspace,
                        stream=None, flags=0):
    """bd_draft_attn over a 4-bit cache."""
    _quant_attn("bd_quant_draft_attn", shape, cache, q, o_out, lse_out, None, idx, count, budget)
    st = (_lib or library()).bd_quant_draft_attn(ctypes.byref(shape), q.data_ptr(), cache._ref, idx.data_ptr(), count.data_ptr(),
                                                 budget, step_j, flags, o_out.data_ptr(), _ptr(lse_out), ws.ptr, ws.nbytes,
                                                 _stream(stream))
    _check("bd_quant_draft_attn", st)


def bd_quant_verify_attn(shape, q, n_q, cache: QuantCache, o_out, lse_out, ws: Workspace, stream=None):
    """bd_verify_attn over a 4-bit cache; n_q = 1 decodes one token."""
    _quant_attn("bd_quant_verify_attn", shape, cache, q, o_out, lse_out, n_q)
    st = (_lib or library()).bd_quant_verify_attn(ctypes.byref(shape), q.data_ptr(), n_q, cache._ref, o_out.data_ptr(), _ptr(lse_out),
                                                  ws.ptr, ws.nbytes, _stream(stream))
    _check("bd_quant_verify_attn", st)


class PagedCache:
    """A pool of pages (the header has the layout): bf16 K and V tensors [n_pages, h_kv, page_size, head_dim] of any strides
    of whole 16 bytes whose rows' elements are adjacent, e.g. x.transpose(1, 2) of an [n_pages, page_size, h_kv, head_dim]
    pool.  The tensors stay the caller's.  Calls take the batch's table of pages beside it: int32 [batch, pages] on the same
    GPU, dense, negative where a page is not there."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape:
            raise ValueError("PagedCache: K and V must be [n_pages, h_kv, page_size, head_dim], alike")
        if k.dtype is not torch.bfloat16 or v.dtype is not torch.bfloat16:
            raise TypeError("PagedCache: K and V are bf16")
        if k.device != v.device:
            raise ValueError("PagedCache: K and V must be on one device")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("PagedCache: the elements of a row must be adjacent")
        self.n_pages, self.h_kv, self.page_size, self.head_dim = (int(x) for x in k.shape)
        if self.head_dim not in (64, 128):
            raise ValueError("PagedCache: head_dim must be 64 or 128")
        if self.page_size < 16 or self.page_size & (self.page_size - 1):
            raise ValueError("PagedCache: page_size must be a power of two, at least 16")
        self.k, self.v = k, v
        self._struct = BdPagedCache(k.data_ptr(), v.data_ptr(), (ctypes.c_int64 * 3)(*k.stride()[:3]),
                                    (ctypes.c_int64 * 3)(*v.stride()[:3]), self.n_pages, self.page_size)
        self.is_cuda = k.is_cuda
        self._gpu = k.get_device() if self.is_cuda else None

    @classmethod
    def empty(cls, n_pages, h_kv, page_size, head_dim, device="cuda"):
        """A pool whose pages are not written yet."""
        return cls(*(torch.empty(n_pages, h_kv, page_size, head_dim, dtype=torch.bfloat16, device=device) for _ in "kv"))

    def shape(self, batch: int, h_q: int, t_ctx: int, t_cap: int, seq_lens=None) -> BdShape:
        return make_shape(batch, h_q, self.h_kv, self.head_dim, t_ctx, t_cap, seq_lens)

    @property
    def nbytes(self) -> int:
        return 2 * self.k.numel() * 2


class Rope:
    """The rotation of rows to their positions (the header's bd_rope).  inv_freq: the angular frequency of each pair of a
    row's first 2 * len(inv_freq) elements (a tensor or a sequence, taken in 64 bits); interleaved: pairs are elements
    (2 j, 2 j + 1), else (j, j + dim / 2); scale: a factor on the rotated rows (a long-context method's)."""

    def __init__(self, inv_freq, interleaved=False, scale=1.0, device=None):
        if device is None:
            device = inv_freq.device if isinstance(inv_freq, torch.Tensor) and inv_freq.is_cuda else "cuda"
        freq = torch.as_tensor(inv_freq, dtype=torch.float64).cpu()
        if freq.dim() != 1 or freq.numel() == 0 or freq.numel() % 8 or freq.numel() > 64:
            raise ValueError("Rope: inv_freq must hold a frequency for each of 8, 16, ... 64 pairs")
        if not torch.isfinite(freq).all() or not math.isfinite(scale):
            raise ValueError("Rope: frequencies and scale must be finite")
        turns = [_turns(w) for w in freq.tolist()]
        self.turns = torch.tensor([x - 2**64 if x >= 2**63 else x for x in turns], dtype=torch.int64, device=device)
        self.dim, self.interleaved, self.scale = 2 * freq.numel(), bool(interleaved), float(scale)
        self._struct = BdRope(self.turns.data_ptr(), self.dim, int(self.interleaved), self.scale)
        self._gpu = self.turns.get_device() if self.turns.is_cuda else None

    @classmethod
    def of_base(cls, dim, base=10000.0, **kw):
        """Pair j of dim / 2 turns by base^(-2 j / dim) a position."""
        return cls([base ** (-2.0 * j / dim) for j in range(dim // 2)], **kw)


# 2^160 / (2 pi), from 2 pi to 35 digits: a frequency of 64 bits keeps all of them
_PER_RADIAN = (10**35 << 160) // 628318530717958647692528676655900577


def _turns(w):
    """w / (2 pi) * 2^64 modulo 2^64, rounded once."""
    m, e = math.frexp(w)
    x, down = int(m * 2**53) * _PER_RADIAN, 149 - e
    return ((x + (1 << down - 1)) >> down if down > 0 else x << -down) % 2**64


# As above: what the calls check is checked once, and told apart only when something does not fit.
def _refuse_paged(name, shape, cache, table, rows=(), row_starts=None, rope=None, **tensors):
    """rows: (tensor, shape, dtypes) of an append or a read."""
    b, _, h, d, _, _ = _shape_ints(shape)
    if (h, d) != (cache.h_kv, cache.head_dim):
        _refuse_cache(name, shape)
    if table.dtype is not _I32:
        raise TypeError(f"{name}: the table must be int32, got {table.dtype}")
    if table.dim() != 2 or table.shape[0] != b or not table.is_contiguous():
        raise ValueError(f"{name}: the table must be a contiguous [{b}, pages] tensor, got {tuple(table.shape)}")
    for t, want, dtypes in rows:
        if t is None:
            continue
        if t.dtype not in dtypes:
            raise TypeError(f"{name}: rows must be {' or '.join('bf16' if x is _BF16 else 'fp32' for x in dtypes)}, got {t.dtype}")
        if t.shape != want:
            raise ValueError(f"{name}: rows must be {tuple(want)}, got {tuple(t.shape)}")
        if t.stride(-1) != 1:
            raise ValueError(f"{name}: the elements of a row must be adjacent")
    if row_starts is not None and (row_starts.dtype is not _I32 or row_starts.shape != (b + 1,) or not row_starts.is_contiguous()):
        _refuse(name, row_starts=(row_starts, _I32, (b + 1,)))
    if rope is not None and rope.dim > d:
        raise ValueError(f"{name}: the rotation must be of at most head_dim elements")
    _refuse(name, **tensors)


_pack_strides = struct.Struct("4q").pack          # (the last one, of a row's elements, goes unread)


def _paged_rows(t, want, dtype, gpu):
    """Pointer and strides (None where they are dense) of rows that fit, else None."""
    if t is None:
        return None, None
    if t.shape == want and t.dtype is dtype and t.get_device() == gpu:
        if t.is_contiguous():
            return t.data_ptr(), None
        st = t.stride()
        if st[-1] == 1:
            return t.data_ptr(), _pack_strides(*st) if len(st) == 4 else _pack_strides(0, *st)
    return None


_device, _raw_stream = (getattr(torch._C, x, None) for x in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


def bd_paged_append(shape, q_rows, k_rows, v_rows, rope, cache: PagedCache, table, q_out, row_starts=None, stream=None):
    """New tokens join a paged cache behind each sequence's context: queries and keys are rotated to their positions (rope: a
    Rope, or None), keys and values written into their pages, queries into q_out (bf16).  Rows are [batch, heads, n,
    head_dim], or with row_starts (int32 [batch + 1] on the GPU) packed [heads, rows, head_dim]; bf16 or fp32, any strides
    of whole 16 bytes; any of q_rows (with q_out), k_rows and v_rows may be None.  q_out may be a bf16 q_rows itself."""
    b, h_q, h, d, _, _ = _shape_ints(shape)
    gpu = cache._gpu
    first = q_rows if q_rows is not None else k_rows if k_rows is not None else v_rows
    if first is None:
        raise ValueError("bd_paged_append: rows of queries, keys or values")
    if (q_rows is None) != (q_out is None):
        raise ValueError("bd_paged_append: q_rows and q_out come together")
    dtype, size = first.dtype, first.shape
    if len(size) != (4 if row_starts is None else 3):
        raise ValueError(f"bd_paged_append: rows must be [batch, heads, n, head_dim], packed [heads, rows, head_dim], got {tuple(size)}")
    n = size[-2]
    if row_starts is None:
        want_q, want_kv = (b, h_q, n, d), (b, h, n, d)
    else:
        want_q, want_kv = (h_q, n, d), (h, n, d)
    ts = table.shape
    q, k = _paged_rows(q_rows, want_q, dtype, gpu), _paged_rows(k_rows, want_kv, dtype, gpu)
    v, o = _paged_rows(v_rows, want_kv, dtype, gpu), _paged_rows(q_out, want_q, _BF16, gpu)
    if not (h == cache.h_kv and d == cache.head_dim and (dtype is _BF16 or dtype is _F32) and q and k and v and o
            and table.dtype is _I32 and len(ts) == 2 and ts[0] == b and table.is_contiguous() and table.get_device() == gpu
            and (rope is None or (rope._gpu == gpu and rope.dim <= d))
            and (row_starts is None or (row_starts.dtype is _I32 and row_starts.shape == (b + 1,) and row_starts.is_contiguous()
                                        and row_starts.get_device() == gpu))):
        kinds = (_BF16, _F32) if dtype not in (_BF16, _F32) else (dtype,)
        _refuse_paged("bd_paged_append", shape, cache, table, ((q_rows, want_q, kinds), (k_rows, want_kv, kinds), (v_rows, want_kv, kinds),
                                                               (q_out, want_q, (_BF16,))), row_starts, rope)
    if _device() != gpu:                       # (the call with the cache's GPU current)
        with torch.cuda.device(gpu):
            return bd_paged_append(shape, q_rows, k_rows, v_rows, rope, cache, table, q_out, row_starts, stream)
    st = (_lib or library()).bd_paged_append(
        shape, n, 1 if dtype is _BF16 else 2, q[0], q[1], k[0], k[1], v[0], v[1],
        None if row_starts is None else row_starts.data_ptr(),
        None if rope is None else rope._struct, cache._struct, table.data_ptr(), ts[1], o[0], o[1],
        _raw_stream(gpu) if stream is None else _stream(stream))
    if st:
        _check("bd_paged_append", st)


def bd_paged_read(shape, cache: PagedCache, table, k_out, v_out=None, first_row=None, stream=None):
    """Reads the context's rows first_row .. first_row + n - 1 (None: those behind the context) into bf16 [batch, h_kv, n,
    head_dim] tensors; either may be None.  Rows of positions at or past a sequence's length are left as they were, those whose
    page is not there are zeros."""
    b, _, h, d, _, _ = _shape_ints(shape)
    gpu = cache._gpu
    first = k_out if k_out is not None else v_out
    if first is None:
        raise ValueError("bd_paged_read: K rows, V rows or both")
    if first_row is None:
        first_row = BD_PAGED_BLOCK_ROWS
    elif first_row < 0:
        raise ValueError("bd_paged_read: first_row must not be negative")
    want = (b, h, first.shape[2] if first.dim() == 4 else -1, d)
    ts = table.shape
    k, v = _paged_rows(k_out, want, _BF16, gpu), _paged_rows(v_out, want, _BF16, gpu)
    if not (h == cache.h_kv and d == cache.head_dim and k and v and table.dtype is _I32 and len(ts) == 2 and ts[0] == b
            and table.is_contiguous() and table.get_device() == gpu):
        _refuse_paged("bd_paged_read", shape, cache, table, ((k_out, want, (_BF16,)), (v_out, want, (_BF16,))))
    if _device() != gpu:                       # (the call with the cache's GPU current)
        with torch.cuda.device(gpu):
            return bd_paged_read(shape, cache, table, k_out, v_out, None if first_row == BD_PAGED_BLOCK_ROWS else first_row, stream)
    st = (_lib or library()).bd_paged_read(
        shape, first_row, want[2], cache._struct, table.data_ptr(), ts[1], k[0], k[1], v[0], v[1],
        _raw_stream(gpu) if stream is None else _stream(stream))
    if st:
        _check("bd_paged_read", st)


def bd_paged_keys(shape, cache: PagedCache, table, k_out, stream=None):
    """Reads the keys of positions 0 .. n - 1 into a bf16 [batch, h_kv, n, head_dim] tensor as bd_select_budget takes them: those
    whose page is not there are NaN, which counts as score 0.  Rows of positions at or past a sequence's length are left as
    they were."""
    b, _, h, d, _, _ = _shape_ints(shape)
    gpu = cache._gpu
    want, ts = (b, h, k_out.shape[2] if k_out.dim() == 4 else -1, d), table.shape
    k = _paged_rows(k_out, want, _BF16, gpu)
    if not (h == cache.h_kv and d == cache.head_dim and k and table.dtype is _I32 and len(ts) == 2 and ts[0] == b
            and table.is_contiguous() and table.get_device() == gpu):
        _refuse_paged("bd_paged_keys", shape, cache, table, ((k_out, want, (_BF16,)),))
    if _device() != gpu:                       # (the call with the cache's GPU current)
        with torch.cuda.device(gpu):
            return bd_paged_keys(shape, cache, table, k_out, stream)
    st = (_lib or library()).bd_paged_keys(
        shape, want[2], cache._struct, table.data_ptr(), ts[1], k[0], k[1], _raw_stream(gpu) if stream is None else _stream(stream))
    if st:
        _check("bd_paged_keys", st)


def bd_paged_verify_attn(shape, q, n_q, cache: PagedCache, table, o_out, lse_out, ws: Workspace, stream=None):
    """bd_verify_attn over a paged cache; n_q = 1 decodes one token."""
    b, h_q, h, d, _, _ = _shape_ints(shape)
    gpu, want, ts = cache._gpu, (b, h_q, n_q, d), table.shape
    if not (h == cache.h_kv and d == cache.head_dim and q.shape == want and o_out.shape == want and q.dtype is _BF16
            and o_out.dtype is _BF16 and q.is_contiguous() and o_out.is_contiguous() and q.get_device() == gpu
            and o_out.get_device() == gpu and ws.buf.get_device() == gpu
            and table.dtype is _I32 and len(ts) == 2 and ts[0] == b and table.is_contiguous() and table.get_device() == gpu
            and (lse_out is None or (lse_out.dtype is _F32 and lse_out.shape == want[:-1] and lse_out.is_contiguous()
                                     and lse_out.get_device() == gpu))):
        _refuse_paged("bd_paged_verify_attn", shape, cache, table, q=(q, _BF16, want), o_out=(o_out, _BF16, want),
                      lse_out=(lse_out, _F32, want[:-1]))
    if _device() != gpu:                       # (the call with the cache's GPU current)
        with torch.cuda.device(gpu):
            return bd_paged_verify_attn(shape, q, n_q, cache, table, o_out, lse_out, ws, stream)
    st = (_lib or library()).bd_paged_verify_attn(
        shape, q.data_ptr(), n_q, cache._struct, table.data_ptr(), ts[1], o_out.data_ptr(),
        None if lse_out is None else lse_out.data_ptr(), ws.buf.data_ptr(), ws.nbytes,
        _raw_stream(gpu) if stream is None else _stream(stream))
    if st:
        _check("bd_paged_verify_attn", st)


def bd_paged_draft_attn(shape, q, cache: PagedCache, table, idx, count, budget, step_j, o_out, lse_out, ws: Workspace,
                        stream=None, flags=0):
    """bd_draft_attn over a paged cache."""
    b, h_q, h, d, _, _ = _shape_ints(shape)
    gpu, want, ts = cache._gpu, (b, h_q, d), table.shape
    if not (h == cache.h_kv and d == cache.head_dim and q.shape == want and o_out.shape == want and q.dtype is _BF16
            and o_out.dtype is _BF16 and q.is_contiguous() and o_out.is_contiguous() and q.get_device() == gpu
            and o_out.get_device() == gpu and ws.buf.get_device() == gpu
            and idx.dtype is _I32 and idx.shape == (b, h, budget) and idx.is_contiguous() and idx.get_device() == gpu
            and count.dtype is _I32 and count.shape == (b, h) and count.is_contiguous() and count.get_device() == gpu
            and table.dtype is _I32 and len(ts) == 2 and ts[0] == b and table.is_contiguous() and table.get_device() == gpu
            and (lse_out is None or (lse_out.dtype is _F32 and lse_out.shape == (b, h_q) and lse_out.is_contiguous()
                                     and lse_out.get_device() == gpu))):
        _refuse_paged("bd_paged_draft_attn", shape, cache, table, q=(q, _BF16, want), o_out=(o_out, _BF16, want),
                      lse_out=(lse_out, _F32, (b, h_q)), idx=(idx, _I32, (b, h, budget)), count=(count, _I32, (b, h)))
    if _device() != gpu:                       # (the call with the cache's GPU current)
        with torch.cuda.device(gpu):
            return bd_paged_draft_attn(shape, q, cache, table, idx, count, budget, step_j, o_out, lse_out, ws, stream, flags)
    st = (_lib or library()).bd_paged_draft_attn(
        shape, q.data_ptr(), cache._struct, table.data_ptr(), ts[1], idx.data_ptr(), count.data_ptr(), budget, step_j,
        flags, o_out.data_ptr(), None if lse_out is None else lse_out.data_ptr(), ws.buf.data_ptr(), ws.nbytes,
        _raw_stream(gpu) if stream is None else _stream(stream))
    if st:
        _check("bd_paged_draft_attn", st)


def bd_check_wait_timeout(ws: Workspace, limit_us: int, stream=None):
    """Runs the bounded-wait error path once (see the header); read the result with
    bd_workspace_status."""
    _check("bd_check_wait_timeout", library().bd_check_wait_timeout(ws.ptr, ws.nbytes, int(limit_us), _stream(stream)))


def bd_workspace_status(ws: Workspace, stream=None) -> int:
    return ws.status(stream)
