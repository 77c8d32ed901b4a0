"""Thin ctypes binding of libbudgetdraft (include/budgetdraft.h).

Argument marshalling only: every computation runs in the library's CUDA kernels.  torch
tensors provide device memory and the current CUDA stream.  There is no fallback: if
the library is not built, or an argument is rejected, these functions raise.
"""

from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch

from .build import LIB_PATH

BD_OK = 0
BD_ERR_CUDA = -5
BD_OP_SELECT, BD_OP_DRAFT, BD_OP_VERIFY, BD_OP_QUANT_DRAFT, BD_OP_QUANT_VERIFY = 1, 2, 3, 4, 5
BD_QUANT_BLOCK_ROWS = -1
BD_QUANT_GROUP = 32
BD_DRAFT_VIEW_READY = 1
BD_SELECT_WINDOW_READY = 1
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


class BudgetDraftError(RuntimeError):
    def __init__(self, func, status):
        self.status = status
        super().__init__(f"{func} failed: {bd_strerror(status)} ({status})")


_lib = None
_P = ctypes.c_void_p
_SHAPE = ctypes.POINTER(BdShape)
_QCACHE = ctypes.POINTER(BdQuantCache)
_STRIDES = ctypes.POINTER(ctypes.c_int64)
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


def bd_check_wait_timeout(ws: Workspace, limit_us: int, stream=None):
    """Runs the bounded-wait error path once (see the header); read the result with
    bd_workspace_status."""
    _check("bd_check_wait_timeout", library().bd_check_wait_timeout(ws.ptr, ws.nbytes, int(limit_us), _stream(stream)))


def bd_workspace_status(ws: Workspace, stream=None) -> int:
    return ws.status(stream)
