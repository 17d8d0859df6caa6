"""Rotary positions with per-head norms, and the paged key / value cache: appending to it, attention over it, the weights
that its rows gather, eviction by them (``skipffn_rotary_*`` and ``skipffn_paged_*``; see ``include/skipffn.h``)."""
from __future__ import annotations

import ctypes
import operator
from typing import Optional, Sequence

from .binding import BF16, FP32, PATH_DEFAULT, SkipFFNError, _on_device, load_library

PAGED_STATUS_WORDS = 64     # SKIPFFN_PAGED_STATUS_WORDS


class _PagedCache(ctypes.Structure):
    _fields_ = [("heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("path", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_seq", ctypes.c_int32), ("table_width", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("n_pages", ctypes.c_int64), ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("cu_new", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class _RotaryConfig(ctypes.Structure):
    _fields_ = [("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("axes", ctypes.c_int32), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
                ("axis", ctypes.POINTER(ctypes.c_int32)), ("eps", ctypes.c_float)]


def bind(lib: ctypes.CDLL) -> None:
    """Argument types of this module's entry points."""
    vp, i32, i64, f32, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    cache = ctypes.POINTER(_PagedCache)
    for name, res, args in (
            ("skipffn_rotary_create", i32, [ctypes.POINTER(vp), ctypes.POINTER(_RotaryConfig)]),
            ("skipffn_rotary_destroy", None, [vp]),
            ("skipffn_rotary_forward", i32, [vp, i32, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp]),
            ("skipffn_rotary_scratch_bytes", size, [vp]),
            ("skipffn_rotary_backward", i32, [vp, i32, i64] + [vp, i64] * 5 + [vp, vp] + [vp, i64] * 2 + [vp, vp, i32, vp, size, vp]),
            ("skipffn_rotary_append", i32, [vp, cache, i64] + [vp, i64] * 4 + [vp, vp, vp, i64, vp]),
            ("skipffn_paged_append", i32, [cache, i64, vp, i64, vp, i64, vp]),
            ("skipffn_paged_attention_scratch_bytes", size, [cache, i32, i64]),
            ("skipffn_paged_attention", i32, [cache, i32, f32, i64, vp, i64, vp, i64, vp, vp, size, vp]),
            ("skipffn_paged_weights", i32, [cache, i32, f32, i64, vp, i64, vp, vp, vp, i32, vp]),
            ("skipffn_paged_evict", i32, [cache, cache, vp, i32, i32, i32, i32, vp, vp, vp, vp]),
            ("skipffn_paged_poll", i32, [cache, vp, ctypes.POINTER(i32)])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args


def _heads(t, name, dtype, index, tokens, heads, d):
    """(address, token stride) of a [tokens, heads, d] CUDA tensor with contiguous heads, checked."""
    if t.dtype is not dtype or t.get_device() != index:
        raise ValueError(f"{name} must be a {dtype} tensor on cuda:{index}")
    shape = t.shape
    if len(shape) != 3 or shape[0] != tokens or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{name} must have shape [{tokens}, {heads}, {d}], got {list(shape)}")
    ld, sh, sd = t.stride()
    if sd != 1 or (sh != d and heads > 1):
        raise ValueError(f"{name} must have contiguous heads")
    return t.data_ptr(), ld if tokens > 1 else heads * d


def _floats(t, name, shape, index):
    import torch
    if t.dtype is not torch.float32 or t.get_device() != index or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor {list(shape)} on cuda:{index}")
    return t.data_ptr()


def _dtype_of(t, name):
    import torch
    if not t.is_cuda or (t.dtype is not torch.bfloat16 and t.dtype is not torch.float32):
        raise ValueError(f"{name} must be a bf16 or fp32 CUDA tensor")
    return BF16 if t.dtype is torch.bfloat16 else FP32


class PagedCache:
    """A paged key / value cache and the batch that is being answered from it (``skipffn_paged_*``).

    ``k_pages``, ``v_pages``: ``[pages, page_size, heads_kv, head_dim]`` bf16 or fp32 CUDA tensors of equal strides, in any
    memory order with contiguous rows of a head (views of one tensor that holds both, say).  ``page_table``: int32
    ``[n_seq, width]``, the pages of each sequence in order; ``cu_new``: int32 ``[n_seq + 1]`` offsets of each sequence's new
    tokens in the arrays of a call; ``lens``: int32 ``[n_seq]`` rows of each sequence, the new tokens among them as the last
    ones; ``max_new``: the most new tokens a sequence may have (it chooses the kernels: an object of its own for single tokens,
    over the same tensors, is faster).  The three integer tensors live on the device and may be
    changed in place between calls and graph replays.  Work is enqueued on the current torch stream; calls that only
    read the cache may overlap.  Keep the object, and the tensors it was made of, as long as a captured call is replayed."""

    def __init__(self, k_pages, v_pages, page_table, cu_new, lens, max_new: int, path: int = PATH_DEFAULT):
        import torch
        self._torch = torch
        dtype = _dtype_of(k_pages, "k_pages")
        self._lib = load_library()
        if k_pages.dim() != 4 or v_pages.shape != k_pages.shape or v_pages.dtype is not k_pages.dtype or v_pages.stride() != k_pages.stride() \
                or v_pages.device != k_pages.device:
            raise ValueError("k_pages and v_pages must be [pages, page_size, heads_kv, head_dim] of one dtype, device and strides")
        pages, page, hk, d = k_pages.shape
        sp, sr, sh, sd = k_pages.stride()
        if sd != 1 and d > 1:
            raise ValueError("the rows of a head must be contiguous")
        index = k_pages.get_device()
        for t, name, dims in ((page_table, "page_table", 2), (cu_new, "cu_new", 1), (lens, "lens", 1)):
            if t.dtype is not torch.int32 or t.get_device() != index or t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
                raise ValueError(f"{name} must be an int32 tensor of {dims} dimension(s) on {k_pages.device}, its last one contiguous")
        n_seq = lens.shape[0]
        if page_table.shape[0] != n_seq or cu_new.shape[0] != n_seq + 1:
            raise ValueError("page_table, cu_new and lens disagree about the number of sequences")
        self.k_pages, self.v_pages, self.page_table, self.cu_new, self.lens = k_pages, v_pages, page_table, cu_new, lens
        self.dtype, self.heads_kv, self.head_dim, self.page_size, self.n_seq = dtype, hk, d, page, n_seq
        self.max_new = operator.index(max_new)
        self.device, self._index = k_pages.device, index
        self._torch_dtype = k_pages.dtype
        # the kernels report what they find wrong with the integer tensors here (poll)
        self._status = torch.zeros(PAGED_STATUS_WORDS, dtype=torch.int32, device=k_pages.device)
        width = page_table.shape[1]
        self._c = _PagedCache(hk, d, dtype, int(path), page, n_seq, width, self.max_new, pages, k_pages.data_ptr(), v_pages.data_ptr(),
                              sp if pages > 1 else 0, sr if page > 1 else 0, sh if hk > 1 else 0, page_table.data_ptr(),
                              page_table.stride(0) if n_seq > 1 else width, cu_new.data_ptr(), lens.data_ptr(), self._status.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._scratch_bytes = {}
        self._made_on = torch._C._cuda_getCurrentRawStream(index)

    def _on_this_stream(self):
        """Calls on any stream report to the status block: its memory must outlive those calls too."""
        torch = self._torch
        if torch._C._cuda_getCurrentRawStream(self._index) != self._made_on and not torch.cuda.is_current_stream_capturing():
            self._status.record_stream(torch.cuda.current_stream(self.device))

    def append(self, k, v) -> None:
        """Writes the new tokens' keys and values, ``[tokens, heads_kv, head_dim]``, to their rows (``skipffn_paged_append``)."""
        n = k.shape[0]
        args = [_heads(t, name, self._torch_dtype, self._index, n, self.heads_kv, self.head_dim) for t, name in ((k, "k"), (v, "v"))]
        self._on_this_stream()
        st = _on_device(self._lib.skipffn_paged_append, self._index, self._ref, n, *args[0], *args[1])
        if st != 0:
            raise SkipFFNError(st, "skipffn_paged_append")

    def attention(self, q, scale: Optional[float] = None, out=None, lse=None):
        """``(out [tokens, heads_q, head_dim], lse [tokens, heads_q] fp32)`` of the new tokens ``q`` over the cache, their own
        rows included (``skipffn_paged_attention``); ``scale`` defaults to ``head_dim ** -0.5``."""
        if q.dim() != 3:
            raise ValueError("q must have shape [tokens, heads_q, head_dim]")
        n, hq, _ = q.shape
        d = self.head_dim
        aq = _heads(q, "q", self._torch_dtype, self._index, n, hq, d)
        if out is None:
            out = q.new_empty(n, hq, d)
        if lse is None:
            lse = q.new_empty(n, hq, dtype=self._torch.float32)
        ao, al = _heads(out, "out", self._torch_dtype, self._index, n, hq, d), _floats(lse, "lse", (n, hq), self._index)
        nbytes = self._scratch_bytes.get((n, hq))
        if nbytes is None:
            nbytes = self._scratch_bytes[n, hq] = int(self._lib.skipffn_paged_attention_scratch_bytes(self._ref, hq, n))
        scratch = q.new_empty(max(nbytes, 16), dtype=self._torch.uint8)
        self._on_this_stream()
        st = _on_device(self._lib.skipffn_paged_attention, self._index, self._ref, hq, d ** -0.5 if scale is None else float(scale), n, *aq,
                        *ao, al, scratch.data_ptr(), scratch.numel())
        if st != 0:
            raise SkipFFNError(st, "skipffn_paged_attention")
        return out, lse

    def weights(self, q, lse, prior=None, out=None, scale: Optional[float] = None, width: Optional[int] = None):
        """``prior`` (or zero) plus the softmax weight that the new tokens ``q`` give to every cache row, per kv head: fp32
        ``[n_seq, heads_kv, width]``, zero past a sequence's rows (``skipffn_paged_weights``).  ``lse`` is that of
        ``attention``; ``out`` may be ``prior``; ``width`` defaults to prior's, out's or the table's rows."""
        if q.dim() != 3:
            raise ValueError("q must have shape [tokens, heads_q, head_dim]")
        n, hq, _ = q.shape
        if width is None:
            like = prior if prior is not None else out
            width = like.shape[-1] if like is not None else self.page_table.shape[1] * self.page_size
        shape = (self.n_seq, self.heads_kv, operator.index(width))
        aq, al = _heads(q, "q", self._torch_dtype, self._index, n, hq, self.head_dim), _floats(lse, "lse", (n, hq), self._index)
        ap = None if prior is None else _floats(prior, "prior", shape, self._index)
        if out is None:
            out = q.new_empty(*shape, dtype=self._torch.float32)
        ao = _floats(out, "out", shape, self._index)
        self._on_this_stream()
        st = _on_device(self._lib.skipffn_paged_weights, self._index, self._ref, hq, self.head_dim ** -0.5 if scale is None else float(scale),
                        n, *aq, al, ap, ao, shape[2])
        if st != 0:
            raise SkipFFNError(st, "skipffn_paged_weights")
        return out

    def evict(self, weights, budget: int, sinks: int = 0, recent: int = 0, into: Optional["PagedCache"] = None):
        """Keeps at most ``budget`` rows of every sequence and kv head: the first ``sinks``, the last ``recent``, and those with
        the largest ``weights [n_seq, heads_kv, width]``; they move in their order to the front of ``into``'s pages, or of
        their own (``skipffn_paged_evict``).  Returns ``(kept [n_seq, heads_kv, budget] int32, lens [n_seq] int32, weights
        [n_seq, heads_kv, budget])``; the ``lens`` of this object are left as they are.  As ``prior`` of ``weights`` the last need
        columns for the rows that follow: copy them to the front of a wider tensor of zeros."""
        torch = self._torch
        budget = operator.index(budget)
        if weights.dim() != 3:
            raise ValueError("weights must have shape [n_seq, heads_kv, width]")
        width = weights.shape[2]
        aw = _floats(weights, "weights", (self.n_seq, self.heads_kv, width), self._index)
        if into is not None and into._index != self._index:
            raise ValueError("into must be on the same device")
        kept = weights.new_empty(self.n_seq, self.heads_kv, max(budget, 0), dtype=torch.int32)
        lens = weights.new_empty(self.n_seq, dtype=torch.int32)
        new = weights.new_empty(self.n_seq, self.heads_kv, max(budget, 0))
        self._on_this_stream()
        if into is not None:
            into._on_this_stream()
        st = _on_device(self._lib.skipffn_paged_evict, self._index, self._ref, None if into is None else into._ref, aw, width, budget,
                        operator.index(sinks), operator.index(recent), kept.data_ptr(), lens.data_ptr(), new.data_ptr())
        if st != 0:
            raise SkipFFNError(st, "skipffn_paged_evict")
        return kept, lens, new

    def poll(self) -> None:
        """Synchronise the stream and raise if a kernel found the integer tensors at fault."""
        site = ctypes.c_int32(0)
        with self._torch.cuda.device(self._index):
            st = self._lib.skipffn_paged_poll(self._ref, self._torch.cuda.current_stream(self.device).cuda_stream, ctypes.byref(site))
        if st != 0:
            raise SkipFFNError(st, f"skipffn_paged_poll (site {site.value})")


class RotaryQK:
    """Queries and keys normalised per head (RMS norm, with ``gamma``) and rotated by position (``skipffn_rotary_*``).

    ``sections``: frequency pairs of each position axis (text: one axis; images and video: time, height, width), default
    one axis; they sum to ``rotary_dim / 2``.  Frequencies are ``base ** (-p / pairs)`` over all pairs, with ``restart`` over
    the pairs of each section, or the ones given as ``inv_freq``.  ``interleaved``: pairs are neighbouring columns instead of
    (p, p + rotary_dim / 2).  Columns from ``rotary_dim`` (default ``head_dim``) on are not rotated.  Host memory only;
    serves every stream, dtype and device."""

    def __init__(self, heads_q: int, heads_kv: int, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0,
                 sections: Optional[Sequence[int]] = None, restart: bool = False, inv_freq: Optional[Sequence[float]] = None,
                 interleaved: bool = False, eps: float = 1e-6):
        self._handle = ctypes.c_void_p()
        self._lib = load_library()
        self.heads_q, self.heads_kv, self.head_dim = operator.index(heads_q), operator.index(heads_kv), operator.index(head_dim)
        rot = self.head_dim if rotary_dim is None else operator.index(rotary_dim)
        pairs = max(rot, 0) // 2
        sections = [pairs] if sections is None else [operator.index(n) for n in sections]
        if not sections or any(n < 0 for n in sections) or sum(sections) != pairs:
            raise ValueError(f"sections must sum to rotary_dim / 2 = {pairs}")
        self.axes = len(sections)
        if inv_freq is None:
            inv_freq = [float(base) ** (-p / n) for n in (sections if restart else [pairs]) for p in range(n)]
        inv_freq = [float(f) for f in inv_freq]
        if len(inv_freq) != pairs:
            raise ValueError(f"inv_freq must have rotary_dim / 2 = {pairs} entries")
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
        cfg = _RotaryConfig(self.heads_q, self.heads_kv, self.head_dim, rot, int(bool(interleaved)), self.axes,
                            (ctypes.c_double * max(pairs, 1))(*inv_freq), (ctypes.c_int32 * max(pairs, 1))(*axis), float(eps))
        st = self._lib.skipffn_rotary_create(ctypes.byref(self._handle), ctypes.byref(cfg))
        if st != 0:
            raise SkipFFNError(st, "skipffn_rotary_create")
        self.rotary_dim = rot
        self._scratch_bytes = int(self._lib.skipffn_rotary_scratch_bytes(self._handle))

    def __del__(self):
        handle, self._handle = getattr(self, "_handle", None), None
        if handle is not None and handle.value:
            self._lib.skipffn_rotary_destroy(handle)

    def _inputs(self, q, k, positions, gamma_q, gamma_k):
        """Checked addresses and strides: q, k, positions, gammas."""
        import torch
        _dtype_of(q, "q")
        n, index, d = q.shape[0], q.get_device(), self.head_dim
        args = _heads(q, "q", q.dtype, index, n, self.heads_q, d) + _heads(k, "k", q.dtype, index, n, self.heads_kv, d)
        if self.rotary_dim:
            if positions is None:
                raise ValueError("positions are needed unless rotary_dim is 0")
            if positions.dim() == 1:
                positions = positions[None]
            if positions.dtype is not torch.int32 or positions.get_device() != index or positions.dim() != 2 \
                    or tuple(positions.shape) != (self.axes, n) or (n > 1 and positions.stride(1) != 1):
                raise ValueError(f"positions must be an int32 tensor [{self.axes}, {n}] on {q.device}, contiguous along the tokens")
            args += positions.data_ptr(), positions.stride(0) if self.axes > 1 else n
        else:
            args += None, 0
        for g, name in ((gamma_q, "gamma_q"), (gamma_k, "gamma_k")):
            if g is not None and (g.dtype is not q.dtype or g.get_device() != index or tuple(g.shape) != (d,) or not g.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous {q.dtype} tensor [{d}] on {q.device}")
        if (gamma_q is None) != (gamma_k is None):
            raise ValueError("gamma_q and gamma_k: both or neither")
        return n, index, args, (None, None) if gamma_q is None else (gamma_q.data_ptr(), gamma_k.data_ptr())

    def forward(self, q, k, positions, gamma_q=None, gamma_k=None, out_q=None, out_k=None):
        """``(q', k')`` of ``q [tokens, heads_q, head_dim]`` and ``k [tokens, heads_kv, head_dim]`` (slices of one fused projection
        need no copy); ``positions`` int32 ``[axes, tokens]`` (``[tokens]`` for one axis).  ``out_q`` may be ``q``, ``out_k`` ``k``."""
        n, index, args, gammas = self._inputs(q, k, positions, gamma_q, gamma_k)
        d = self.head_dim
        out_q = q.new_empty(n, self.heads_q, d) if out_q is None else out_q
        out_k = q.new_empty(n, self.heads_kv, d) if out_k is None else out_k
        st = _on_device(self._lib.skipffn_rotary_forward, index, self._handle, _dtype_of(q, "q"), n, *args, *gammas,
                        *_heads(out_q, "out_q", q.dtype, index, n, self.heads_q, d), *_heads(out_k, "out_k", q.dtype, index, n, self.heads_kv, d))
        if st != 0:
            raise SkipFFNError(st, "skipffn_rotary_forward")
        return out_q, out_k

    def backward(self, dout_q, dout_k, q, k, positions, gamma_q=None, gamma_k=None, dq=None, dk=None, dw_fp32: bool = False):
        """``(dq, dk, dgamma_q, dgamma_k)`` from the gradients of ``forward``'s results and its inputs; the last two are None
        without gammas.  ``dq`` may be ``dout_q`` or ``q``, ``dk`` likewise."""
        import torch
        n, index, args, gammas = self._inputs(q, k, positions, gamma_q, gamma_k)
        d, dt = self.head_dim, q.dtype
        up = _heads(dout_q, "dout_q", dt, index, n, self.heads_q, d) + _heads(dout_k, "dout_k", dt, index, n, self.heads_kv, d)
        dq = q.new_empty(n, self.heads_q, d) if dq is None else dq
        dk = q.new_empty(n, self.heads_kv, d) if dk is None else dk
        dgq = dgk = None
        small = (None, None, 0, None, 0)
        if gamma_q is not None:
            gdt = torch.float32 if dw_fp32 else dt
            dgq, dgk = q.new_empty(d, dtype=gdt), q.new_empty(d, dtype=gdt)
            scratch = q.new_empty(self._scratch_bytes, dtype=torch.uint8)
            small = (dgq.data_ptr(), dgk.data_ptr(), int(bool(dw_fp32)), scratch.data_ptr(), self._scratch_bytes)
        st = _on_device(self._lib.skipffn_rotary_backward, index, self._handle, _dtype_of(q, "q"), n, *up, *args, *gammas,
                        *_heads(dq, "dq", dt, index, n, self.heads_q, d), *_heads(dk, "dk", dt, index, n, self.heads_kv, d), *small)
        if st != 0:
            raise SkipFFNError(st, "skipffn_rotary_backward")
        return dq, dk, dgq, dgk

    def append(self, cache: PagedCache, q, k, v, positions, gamma_q=None, gamma_k=None, out_q=None):
        """``q'`` of the new tokens of ``cache``'s batch; ``k'`` and ``v`` go to their rows of the cache
        (``skipffn_rotary_append``)."""
        n, index, args, gammas = self._inputs(q, k, positions, gamma_q, gamma_k)
        if index != cache._index or q.dtype is not cache._torch_dtype:
            raise ValueError(f"q must be a {cache._torch_dtype} tensor on {cache.device}")
        d = self.head_dim
        out_q = q.new_empty(n, self.heads_q, d) if out_q is None else out_q
        cache._on_this_stream()
        st = _on_device(self._lib.skipffn_rotary_append, index, self._handle, cache._ref, n, *args[:4],
                        *_heads(v, "v", q.dtype, index, n, self.heads_kv, d), *args[4:], *gammas,
                        *_heads(out_q, "out_q", q.dtype, index, n, self.heads_q, d))
        if st != 0:
            raise SkipFFNError(st, "skipffn_rotary_append")
        return out_q
