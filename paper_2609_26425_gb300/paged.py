"""Rotary positions over three axes and the uncompressed, paged side of the
cache (binding of the qwm_rope* and qwm_paged* entry points of include/qwm.h).

Like the rest of the binding this only marshals arguments: it checks dtypes,
shapes, strides and devices, passes device pointers and the current stream, and
uses PyTorch for device memory.  ``Rope`` holds a rotation's frequencies,
``PagedCache`` the pages, ``PagedBatch`` the sequences of a step; the calls are
qwm_rope, qwm_rope_backward, qwm_paged_append and qwm_paged_attend.
"""
from __future__ import annotations

import ctypes as ct
import math

import torch

_P = ct.c_void_p
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


class QwmRows(ct.Structure):
    _fields_ = [("data", _P), ("token_stride", ct.c_int64), ("head_stride", ct.c_int64), ("heads", ct.c_int32)]


class QwmRopeConfig(ct.Structure):
    _fields_ = [("head_dim", ct.c_int32), ("dtype", ct.c_int32), ("pairs", ct.c_int32 * 3),
                ("interleaved", ct.c_int32)]


class QwmPagedConfig(ct.Structure):
    _fields_ = [("kv_heads", ct.c_int32), ("head_dim", ct.c_int32), ("page_tokens", ct.c_int32),
                ("dtype", ct.c_int32), ("num_pages", ct.c_int64)]


class QwmPagedBatch(ct.Structure):
    _fields_ = [("num_seqs", ct.c_int32), ("table_stride", ct.c_int32), ("max_q", ct.c_int32),
                ("max_kv", ct.c_int32), ("tokens", ct.c_int64), ("q_offsets", _P), ("kv_len", _P),
                ("page_table", _P)]


class QwmMask(ct.Structure):
    _fields_ = [("block", ct.c_int32), ("window", ct.c_int32), ("sinks", ct.c_int32)]


_ROWS = ct.POINTER(QwmRows)
_ROPE = ct.POINTER(QwmRopeConfig)
_BATCH = ct.POINTER(QwmPagedBatch)
_MASK = ct.POINTER(QwmMask)


_C = None  # the loaded library, argument types declared


def declare(L):
    """Argument types of the entry points in the loaded library."""
    global _C
    rope = [_ROPE, _P, _P, ct.c_int64, _ROWS, _ROWS, _ROWS, _ROWS, _P]
    for name, args, res in (
            ("qwm_rope", rope, ct.c_int), ("qwm_rope_backward", rope, ct.c_int),
            ("qwm_paged_bytes", [ct.POINTER(QwmPagedConfig)], ct.c_size_t),
            ("qwm_paged_init", [ct.POINTER(_P), ct.POINTER(QwmPagedConfig), _P, ct.c_size_t, _P], ct.c_int),
            ("qwm_paged_free", [_P], None),
            ("qwm_paged_status", [_P, ct.POINTER(ct.c_int32), _P], ct.c_int),
            ("qwm_paged_set_wait_limit", [_P, ct.c_uint64], ct.c_int),
            ("qwm_paged_set_idle_role", [_P, ct.c_int32], ct.c_int),
            ("qwm_paged_append", [_P, _BATCH, _ROWS, _ROWS, _ROPE, _P, _P, _ROWS, _ROWS, _P], ct.c_int),
            ("qwm_paged_attend_workspace_bytes", [_P, _BATCH, ct.c_int32, _MASK], ct.c_size_t),
            ("qwm_paged_attend", [_P, _BATCH, _ROWS, _MASK, ct.c_float, _ROWS, _P, _P, ct.c_size_t, _P],
             ct.c_int)):
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, res
    _C = L


def _lib():
    if _C is None:
        from . import lib
        lib()
    return _C


def _check(fn, st):
    if st:
        from . import QwmError
        raise QwmError(fn, st)


_raw_stream = torch._C._cuda_getCurrentRawStream  # current stream of a device, without a Stream object


def _rows(t, dtype, name, tokens=None, head_dim=None):
    """A [tokens][heads][head_dim] tensor as qwm_rows (any strides of tokens and heads)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype):
        raise ValueError(f"{name} must be a {dtype} CUDA tensor")
    shape = t.shape
    if len(shape) != 3 or (tokens is not None and shape[0] != tokens) or (
            head_dim is not None and shape[2] != head_dim):
        raise ValueError(f"{name} has shape {tuple(shape)}, expected ({tokens}, heads, {head_dim})")
    st, sh, sc = t.stride()
    if sc != 1:
        raise ValueError(f"{name} must have contiguous channels")
    n, h, _ = shape  # the stride of a dimension of one is never used
    return QwmRows(t.data_ptr(), st if n > 1 else 0, sh if h > 1 else 0, h)


def _out(like, out, name):
    """An output with the shape and dtype of `like`: the caller's, or a new contiguous tensor."""
    if out is None:
        out = torch.empty_like(like) if like.is_contiguous() else torch.empty(like.shape, dtype=like.dtype,
                                                                              device=like.device)
        _, h, d = like.shape
        return out, QwmRows(out.data_ptr(), h * d, d, h)
    if out.shape != like.shape:
        raise ValueError(f"{name} has shape {tuple(out.shape)}, expected {tuple(like.shape)}")
    return out, _rows(out, like.dtype, name)


def _ints(t, shape, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.int32 and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    return t


def _stream(t):
    return _raw_stream(t.get_device())


# ------------------------------------------------------------------ rope
class Rope:
    """A rotation over three axes: fp32 frequencies ``inv_freq`` [P] on the GPU,
    ``pairs`` = (time, height, width) pairs that sum to P, and the layout of a
    pair's two channels (neighbours, or halves of the rotated part)."""

    def __init__(self, inv_freq, pairs, interleaved=True):
        pairs = tuple(int(p) for p in pairs)
        if len(pairs) != 3 or min(pairs) < 0:
            raise ValueError("pairs must be three counts (time, height, width)")
        if not (isinstance(inv_freq, torch.Tensor) and inv_freq.is_cuda and inv_freq.dtype == torch.float32
                and inv_freq.is_contiguous() and tuple(inv_freq.shape) == (sum(pairs),)):
            raise ValueError(f"inv_freq must be a contiguous fp32 CUDA tensor [{sum(pairs)}]")
        self.inv_freq, self.pairs, self.interleaved = inv_freq, pairs, bool(interleaved)
        self.freq_ptr = inv_freq.data_ptr()
        self._cfg = {}

    def config(self, head_dim, dtype):
        cfg = self._cfg.get((head_dim, dtype))
        if cfg is None:
            if dtype not in _DTYPES:
                raise ValueError("the rotation takes bf16 or fp16 tensors")
            cfg = QwmRopeConfig(head_dim, _DTYPES[dtype], (ct.c_int32 * 3)(*self.pairs), int(self.interleaved))
            self._cfg[(head_dim, dtype)] = cfg
        return cfg


def _turn(name, rope, q, pos, k, q_out, k_out):
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [tokens][heads][head_dim] tensor")
    n, _, d = q.shape
    cfg = rope.config(d, q.dtype)
    qr = _rows(q, q.dtype, "q")
    q_out, qo = _out(q, q_out, "q_out")
    kr = ko = None
    if k is not None:
        kr = _rows(k, q.dtype, "k", n, d)
        k_out, ko = _out(k, k_out, "k_out")
    st = getattr(_C or _lib(), name)(cfg, rope.freq_ptr, _ints(pos, (n, 3), "pos").data_ptr(), n, qr, qo, kr, ko,
                                     _raw_stream(q.get_device()))
    if st:
        _check(name, st)
    return q_out if k is None else (q_out, k_out)


def qwm_rope(rope: Rope, q, pos, k=None, q_out=None, k_out=None):
    """Queries (and Keys) turned to their positions ``pos`` (int32 [tokens][3]);
    ``q_out=q`` works in place.  Returns q_out, or (q_out, k_out) with Keys."""
    return _turn("qwm_rope", rope, q, pos, k, q_out, k_out)


def qwm_rope_backward(rope: Rope, dq, pos, dk=None, dq_out=None, dk_out=None):
    """Gradient of qwm_rope: the outputs' gradients turned back."""
    return _turn("qwm_rope_backward", rope, dq, pos, dk, dq_out, dk_out)


# ------------------------------------------------------------------ pages
class PagedCache:
    """Pages of bf16 or fp16 Keys and Values in a torch-allocated device buffer;
    ``pages`` is [num_pages][Keys, Values][kv_heads][page_tokens][head_dim]."""

    def __init__(self, kv_heads, num_pages, page_tokens=64, head_dim=128, dtype=torch.bfloat16, device=None):
        if dtype not in _DTYPES:
            raise ValueError("pages hold bf16 or fp16")
        self.cfg = QwmPagedConfig(kv_heads, head_dim, page_tokens, _DTYPES[dtype], num_pages)
        self.dtype, self.head_dim, self.kv_heads, self.page_tokens = dtype, head_dim, kv_heads, page_tokens
        self.num_pages, self.scale = num_pages, 1.0 / math.sqrt(head_dim) if head_dim > 0 else 1.0
        n = int(_lib().qwm_paged_bytes(self.cfg))
        if n == 0:
            _check("qwm_paged_bytes", 2)
        dev = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        raw = torch.empty(n + 1024, dtype=torch.uint8, device=dev)
        off = (-raw.data_ptr()) % 1024
        self.buffer = raw[off:off + n]
        self.pages = self.buffer[256:].view(dtype).view(num_pages, 2, kv_heads, page_tokens, head_dim)
        h = _P()
        _check("qwm_paged_init", _lib().qwm_paged_init(ct.byref(h), self.cfg, self.buffer.data_ptr(), n,
                                                      _stream(self.buffer)))
        self.handle = h

    def __del__(self):
        h = getattr(self, "handle", None)
        if h and _C is not None:
            _C.qwm_paged_free(h)
            self.handle = None

    def set_wait_limit(self, ns: int):
        _check("qwm_paged_set_wait_limit", _lib().qwm_paged_set_wait_limit(self.handle, int(ns)))

    def set_idle_role(self, role: int):
        """qwm_paged_set_idle_role: test hook of the timeout path (0 = normal work)."""
        _check("qwm_paged_set_idle_role", _lib().qwm_paged_set_idle_role(self.handle, int(role)))

    def status(self) -> int:
        """Read and clear the device status word (synchronises the stream)."""
        v = ct.c_int32()
        _check("qwm_paged_status", _lib().qwm_paged_status(self.handle, ct.byref(v), _stream(self.buffer)))
        return v.value


class PagedBatch:
    """The sequences of a step: int32 device tensors ``q_offsets`` [B + 1] (rows
    of each sequence's new tokens), ``kv_len`` [B] (tokens held, the new ones at
    the end) and ``page_table`` [B][pages]; ``max_q`` and ``max_kv`` bound them.
    The tensors may change between calls (a captured graph's step, say) as long
    as the bounds and the number of rows hold."""

    def __init__(self, q_offsets, kv_len, page_table, max_q, max_kv, tokens=None):
        if not isinstance(kv_len, torch.Tensor) or kv_len.dim() != 1:
            raise ValueError("kv_len must be an int32 CUDA tensor [sequences]")
        B = kv_len.shape[0]
        _ints(kv_len, (B,), "kv_len")
        _ints(q_offsets, (B + 1,), "q_offsets")
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
            raise ValueError("page_table must be an int32 CUDA tensor [sequences][pages]")
        _ints(page_table, (B, page_table.shape[1]), "page_table")
        self.tensors = (q_offsets, kv_len, page_table)
        self.num_seqs, self.max_q, self.max_kv = B, int(max_q), int(max_kv)
        self.tokens = tokens
        self._c = {}

    def struct(self, tokens):
        if self.tokens is not None and tokens != self.tokens:
            raise ValueError(f"the batch has {self.tokens} rows, the tensor {tokens}")
        s = self._c.get(tokens)
        if s is None:
            q_offsets, kv_len, table = self.tensors
            s = self._c[tokens] = QwmPagedBatch(self.num_seqs, table.shape[1], self.max_q, self.max_kv, tokens,
                                                q_offsets.data_ptr(), kv_len.data_ptr(), table.data_ptr())
        return s


def qwm_paged_append(cache: PagedCache, batch: PagedBatch, k, v, rope: Rope = None, pos=None, q=None, q_out=None):
    """Store the new tokens' Keys and Values in their pages; with ``rope`` the Keys
    are turned to ``pos`` on the way, and ``q`` is turned beside them.  Returns
    the Queries (a new tensor, or q_out), or None without q."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a [tokens][heads][head_dim] tensor")
    n, d, t = k.shape[0], cache.head_dim, cache.dtype
    kr, vr = _rows(k, t, "k", n, d), _rows(v, t, "v", n, d)
    cfg = freq = at = qr = qo = None
    if rope is not None:
        cfg, freq, at = rope.config(d, t), rope.freq_ptr, _ints(pos, (n, 3), "pos").data_ptr()
    if q is not None:
        qr = _rows(q, t, "q", n, d)
        q_out, qo = _out(q, q_out, "q_out")
    st = (_C or _lib()).qwm_paged_append(cache.handle, batch.struct(n), kr, vr, cfg, freq, at, qr, qo,
                                         _raw_stream(k.get_device()))
    if st:
        _check("qwm_paged_append", st)
    return q_out if q is not None else None


def qwm_paged_attend_workspace_bytes(cache: PagedCache, batch: PagedBatch, q_heads, tokens, window=0, sinks=0,
                                     block=1) -> int:
    return int(_lib().qwm_paged_attend_workspace_bytes(cache.handle, batch.struct(tokens), q_heads,
                                                       QwmMask(block, window, sinks)))


def paged_attend_workspace(cache: PagedCache, batch: PagedBatch, q_heads, window=0, sinks=0, block=1):
    """A zeroed scratch buffer for qwm_paged_attend(..., workspace=), or None when
    none is needed (the size does not depend on the number of rows)."""
    n = qwm_paged_attend_workspace_bytes(cache, batch, q_heads, batch.tokens or 1, window, sinks, block)
    if n == 0:
        return None
    raw = torch.zeros(n + 256, dtype=torch.uint8, device=cache.buffer.device)
    off = (-raw.data_ptr()) % 256
    return raw[off:off + n]


def qwm_paged_attend(cache: PagedCache, batch: PagedBatch, q, window=0, sinks=0, block=1, sm_scale=None, out=None,
                     lse=None, want_lse=False, workspace=None):
    """Attention of the batch's rows over the pages of their sequences: block-causal
    (``block`` tokens a block, 1 = token-causal), the last ``window`` tokens up to
    the end of the row's block (0: all) and the first ``sinks`` tokens."""
    qr = _rows(q, cache.dtype, "q", None, cache.head_dim)
    n, h, _ = q.shape
    out, orows = _out(q, out, "out")
    if lse is not None:
        if not (lse.is_cuda and lse.dtype is torch.float32 and lse.is_contiguous() and lse.shape == (h, n)):
            raise ValueError("lse must be a contiguous fp32 CUDA tensor [heads][tokens]")
    elif want_lse:
        lse = torch.empty((h, n), dtype=torch.float32, device=q.device)
    ws, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.nbytes)
    st = (_C or _lib()).qwm_paged_attend(
        cache.handle, batch.struct(n), qr, QwmMask(block, window, sinks), cache.scale if sm_scale is None else sm_scale,
        orows, None if lse is None else lse.data_ptr(), ws, size, _raw_stream(q.get_device()))
    if st:
        _check("qwm_paged_attend", st)
    return out if lse is None else (out, lse)
