"""Rotary positions over three axes and the uncompressed, paged side of the
cache (binding of the qwm_rope* and qwm_paged* entry points of include/qwm.h).

``Rope`` holds a rotation's frequencies, ``PagedCache`` the pages, ``PagedBatch``
the sequences of a step; the calls are qwm_rope, qwm_rope_backward,
qwm_paged_append and qwm_paged_attend.  Like the rest of the binding these only
marshal arguments (dtypes, shapes, strides and devices are checked, PyTorch is
used for device memory); they go through the compiled csrc/binding.cpp, because
a call for a single token is as long as its binding.  Autograd records qwm_rope; the
paged calls leave no history.
"""
from __future__ import annotations

import ctypes as ct
import importlib.util
import math
import os

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


_B = None  # csrc/binding.cpp


def binding():
    """Load the compiled binding (raises if it has not been built)."""
    global _B
    if _B is None:
        from . import LIB_PATH, QwmError
        _lib()
        path = os.path.join(os.path.dirname(LIB_PATH), "qwm_binding.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        spec = importlib.util.spec_from_file_location("qwm_binding", path)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        mod.set_error(QwmError)
        _B = mod
    return _B


def _check(fn, st):
    if st:
        from . import QwmError
        raise QwmError(fn, st)


def _stream(t):
    return torch.cuda.current_stream(t.device).cuda_stream


def _ints(t, shape, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.int32 and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    return t


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
        self._key = (inv_freq.data_ptr(), *pairs, int(self.interleaved), inv_freq.device.index)


class _Recorded(torch.autograd.Function):
    """The rotation as autograd sees it; its gradient is the rotation back."""

    @staticmethod
    def forward(ctx, rope, back, q, pos, k, q_out, k_out):
        ctx.rope, ctx.back = rope, back
        ctx.save_for_backward(pos, rope.inv_freq)
        ctx.mark_dirty(*(t for t in (q if q_out is True else q_out, k if k_out is True else k_out) if t is not None))
        return binding().turn(back, rope._key, q, pos, k, q if q_out is True else q_out, k if k_out is True else k_out)

    @staticmethod
    def backward(ctx, dq, dk=None):
        pos = ctx.saved_tensors[0]
        need = [g is not None and ctx.needs_input_grad[i] for g, i in ((dq, 2), (dk, 4))]
        given = [_readable(g) for g, n in zip((dq, dk), need) if n]
        turn = qwm_rope if ctx.back else qwm_rope_backward
        got = turn(ctx.rope, given[0], pos, *given[1:]) if given else ()
        got = iter(got if isinstance(got, tuple) else (got,))
        dq, dk = (next(got) if n else None for n in need)
        return None, None, dq, None, dk, None, None


def _readable(g):
    """A gradient in a layout that the kernels read (a sum's, say, has strides of zero)."""
    return g if g.stride(2) == 1 and (g.stride(0) | g.stride(1)) % 8 == 0 and g.data_ptr() % 16 == 0 else g.contiguous()


def _record(rope, back, q, pos, k, q_out, k_out):
    # True: in place (a tensor is passed to autograd once)
    return _Recorded.apply(rope, back, q, pos, k, True if q_out is q else q_out,
                           True if k is not None and k_out is k else k_out)


def qwm_rope(rope: Rope, q, pos, k=None, q_out=None, k_out=None):
    """Queries (and Keys) turned to their positions ``pos`` (int32 [tokens][3]);
    ``q_out=q`` works in place.  Returns q_out, or (q_out, k_out) with Keys.
    Autograd records the call where it is on and q or k requires a gradient
    (``inv_freq`` has none)."""
    got = (_B or binding()).turn(False, rope._key, q, pos, k, q_out, k_out)
    return got if got is not None else _record(rope, False, q, pos, k, q_out, k_out)


def qwm_rope_backward(rope: Rope, dq, pos, dk=None, dq_out=None, dk_out=None):
    """Gradient of qwm_rope: the outputs' gradients turned back."""
    got = (_B or binding()).turn(True, rope._key, dq, pos, dk, dq_out, dk_out)
    return got if got is not None else _record(rope, True, dq, pos, dk, dq_out, dk_out)


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
        with torch.cuda.device(self.buffer.device):    # a default stream's handle is the current device's
            _check("qwm_paged_init", _lib().qwm_paged_init(ct.byref(h), self.cfg, self.buffer.data_ptr(), n,
                                                          _stream(self.buffer)))
        self.handle = h
        self._key = (h.value, head_dim, _DTYPES[dtype], self.buffer.device.index)

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
        with torch.cuda.device(self.buffer.device):
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
        if not q_offsets.device == kv_len.device == page_table.device:
            raise ValueError("q_offsets, kv_len and page_table must be on one device")
        self.tensors = (q_offsets, kv_len, page_table)
        self.num_seqs, self.max_q, self.max_kv = B, int(max_q), int(max_kv)
        self.tokens = tokens
        self._c = QwmPagedBatch(B, page_table.shape[1], self.max_q, self.max_kv, -1 if tokens is None else tokens,
                                q_offsets.data_ptr(), kv_len.data_ptr(), page_table.data_ptr())
        self._key = (ct.addressof(self._c), self._c.tokens, kv_len.device.index)

    def struct(self, tokens):
        """The C descriptor for a call of `tokens` rows."""
        c = QwmPagedBatch.from_buffer_copy(self._c)
        c.tokens = tokens
        return c


def qwm_paged_append(cache: PagedCache, batch: PagedBatch, k, v, rope: Rope = None, pos=None, q=None, q_out=None):
    """Store the new tokens' Keys and Values in their pages; with ``rope`` the Keys
    are turned to ``pos`` on the way, and ``q`` is turned beside them.  Returns
    the Queries (a new tensor, or q_out), or None without q."""
    return (_B or binding()).append(cache._key, batch._key, k, v, None if rope is None else rope._key, pos, q, q_out)


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
    return (_B or binding()).attend(cache._key, batch._key, q, block, window, sinks,
                                    cache.scale if sm_scale is None else sm_scale, out, lse, want_lse, workspace)
