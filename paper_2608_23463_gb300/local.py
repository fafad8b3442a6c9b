"""Attention of the local stream (PyTorch holds memory).

``QKRope`` norms and rotates queries and keys (``pf_qk_rope_*``), ``WindowAttention``
is causal attention in a sliding window with sinks (``pf_window_attn_*``) and
``PagedKVCache`` keeps the keys and values of many sequences in pages
(``pf_paged_*``): ``append`` writes new tokens' rows, ``attend`` is the attention
of every sequence's newest token.  All calls run on the current CUDA stream;
none does arithmetic of its own.  Matrices are 2D tensors whose rows may lie
apart (a slice of a projection's output serves as it is).
"""
from __future__ import annotations

from ctypes import byref
from typing import Optional, Sequence, Tuple

import torch

from . import (PF_BF16, PF_ERR_CAPACITY, PF_ERR_INVALID_ARG, PF_F32, QKV, PagedCache, PagedDesc,
               ProxyFormerError, QKDesc, WindowDesc, _check, _ptr, load, pf_paged_advance,
               pf_paged_attn_workspace_size, pf_qk_rope_workspace_size, pf_window_attn_saved_size,
               pf_window_attn_workspace_size)

# The operators take a few microseconds where a token or two is served, less than a
# call's Python costs: the methods below check their tensors once, fill the C structs
# by position and call the library's function that __init__ looked up.


def _stream(t: torch.Tensor) -> int:
    """The current stream of t's device (torch.cuda.current_stream().cuda_stream, without
    the object: 0.1 us for 2.8)."""
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _rows(name: str, t: torch.Tensor, rows: int, width: int, dtype: torch.dtype) -> int:
    """Checks that the library can take t, a 2D CUDA matrix with its values side by side
    in a row, and returns its leading dimension."""
    if t.dtype is not dtype or t.shape != (rows, width) or not t.is_cuda:
        bad = True
    else:
        ld, one = t.stride()
        bad = one != 1 and width > 1
    if bad:
        raise ProxyFormerError(PF_ERR_INVALID_ARG, f"{name} must be a [{rows}, {width}] {dtype} "
                               "CUDA matrix with contiguous rows")
    return ld if rows > 1 else width  # the stride of a single row says nothing


def _ints(name: str, t: Optional[torch.Tensor], *shape: int) -> Optional[int]:
    """Pointer of an int32 CUDA tensor of that shape, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise ProxyFormerError(PF_ERR_INVALID_ARG, f"{name} must be a contiguous int32 CUDA tensor "
                               f"of shape {list(shape)}")
    return t.data_ptr()


class QKRope:
    """RMSNorm of every query and key head (with weights w_q, w_k [dh]; None: no
    norm) and its position rotation: ``pairs`` pairs of a head for every position
    axis (default: one axis, all of them; (): no rotation)."""

    def __init__(self, n_heads: int, n_kv: int, dh: int, w_q: Optional[torch.Tensor] = None,
                 w_k: Optional[torch.Tensor] = None, pairs: Optional[Sequence[int]] = None,
                 theta: float = 10000.0, eps: float = 1e-6, dtype: torch.dtype = torch.bfloat16):
        pairs = (dh // 2,) if pairs is None else tuple(pairs)
        if len(pairs) > 3 or dtype not in (torch.bfloat16, torch.float32):
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "at most 3 axes; bf16 or fp32")
        for n, w in (("w_q", w_q), ("w_k", w_k)):
            if w is not None and (w.shape != (dh,) or w.dtype != torch.float32
                                  or not w.is_contiguous() or not w.is_cuda):
                raise ProxyFormerError(PF_ERR_INVALID_ARG, f"{n} must be {dh} fp32 values on the GPU")
        self.n_heads, self.n_kv, self.dh, self.dtype, self.n_axes = n_heads, n_kv, dh, dtype, len(pairs)
        self.nq, self.nk = n_heads * dh, n_kv * dh
        self.w_q, self.w_k = w_q, w_k
        self.pw_q, self.pw_k = _ptr(w_q), _ptr(w_k)
        self.desc = QKDesc(n_heads, n_kv, dh, PF_F32 if dtype == torch.float32 else PF_BF16,
                           len(pairs), (pairs + (0, 0, 0))[:3], theta, eps)
        self.ref = byref(self.desc)
        self.fwd, self.bwd = load().pf_qk_rope_fwd, load().pf_qk_rope_bwd
        self.ws: Optional[torch.Tensor] = None

    def _qk(self, rows: int, q: torch.Tensor, k: torch.Tensor) -> QKV:
        lq, lk = _rows("q", q, rows, self.nq, self.dtype), _rows("k", k, rows, self.nk, self.dtype)
        return QKV(q.data_ptr(), k.data_ptr(), None, lq, lk, 0)

    def _new(self, rows: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
        return (torch.empty((rows, self.nq), dtype=self.dtype, device=device),
                torch.empty((rows, self.nk), dtype=self.dtype, device=device))

    def forward(self, q: torch.Tensor, k: torch.Tensor, L: Optional[int] = None,
                pos: Optional[torch.Tensor] = None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """q [rows, n_heads*dh], k [rows, n_kv*dh] -> the same normed and turned (into
        ``out``, a pair, which may be (q, k) itself).  Positions: pos [rows, axes]
        int32, or the row's place in its sequence of L rows (default: one sequence)."""
        rows = q.shape[0]
        x = self._qk(rows, q, k)
        out = self._new(rows, q.device) if out is None else out
        s = self.fwd(self.ref, rows, L or max(rows, 1), byref(x), self.pw_q, self.pw_k,
                     _ints("pos", pos, rows, self.n_axes), byref(self._qk(rows, *out)), _stream(q))
        if s:
            _check(s)
        return out

    def backward(self, q: torch.Tensor, k: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                 L: Optional[int] = None, pos: Optional[torch.Tensor] = None, out=None):
        """From the forward's inputs and the gradients of its results: the gradients
        of q and k (into ``out``, which may be (dq, dk) itself) and of w_q and w_k
        (None without them)."""
        rows = q.shape[0]
        x, g = self._qk(rows, q, k), self._qk(rows, dq, dk)
        out = self._new(rows, q.device) if out is None else out
        dw_q, dw_k = (None if w is None else torch.empty_like(w) for w in (self.w_q, self.w_k))
        if self.ws is None and (dw_q is not None or dw_k is not None):
            self.ws = torch.empty(pf_qk_rope_workspace_size(self.desc), dtype=torch.uint8,
                                  device=q.device)
        s = self.bwd(self.ref, rows, L or max(rows, 1), byref(x), self.pw_q, self.pw_k,
                     _ints("pos", pos, rows, self.n_axes), byref(g), byref(self._qk(rows, *out)),
                     _ptr(dw_q), _ptr(dw_k), _ptr(self.ws), 0 if self.ws is None else self.ws.numel(),
                     _stream(q))
        if s:
            _check(s)
        return (*out, dw_q, dw_k)


class WindowAttention:
    """Causal attention of ``batch`` sequences of L rows: row i sees the last ``window``
    rows up to itself (0: all) and the first ``n_sink``.  bf16, head width 64."""

    def __init__(self, batch: int, L: int, n_heads: int, n_kv: int, dh: int = 64, window: int = 0,
                 n_sink: int = 0):
        self.rows, self.nq, self.nk = batch * L, n_heads * dh, n_kv * dh
        self.desc = WindowDesc(batch, L, n_heads, n_kv, dh, window, n_sink)
        self.ref = byref(self.desc)
        self.fwd, self.bwd = load().pf_window_attn_fwd, load().pf_window_attn_bwd
        self.saved_size = pf_window_attn_saved_size(self.desc)
        self.saved: Optional[torch.Tensor] = None  # of the last forward for training
        self.ws: Optional[torch.Tensor] = None

    def _qkv(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> QKV:
        n, bf = self.rows, torch.bfloat16
        ld = (_rows("q", q, n, self.nq, bf), _rows("k", k, n, self.nk, bf),
              _rows("v", v, n, self.nk, bf))
        return QKV(q.data_ptr(), k.data_ptr(), v.data_ptr(), *ld)

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, train: bool = True,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q [batch*L, n_heads*dh], k, v [batch*L, n_kv*dh] -> [batch*L, n_heads*dh];
        ``train`` keeps what the backward needs beside them."""
        x, bf, dev = self._qkv(q, k, v), torch.bfloat16, q.device
        out = torch.empty((self.rows, self.nq), dtype=bf, device=dev) if out is None else out
        if train:  # a new buffer: the last forward's may still be read on another stream
            self.saved = torch.empty(self.saved_size, dtype=torch.uint8, device=dev)
        s = self.fwd(self.ref, byref(x), out.data_ptr(), _rows("out", out, self.rows, self.nq, bf),
                     self.saved.data_ptr() if train else None, _stream(q))
        if s:
            _check(s)
        return out

    def backward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                 dout: torch.Tensor, saved: Optional[torch.Tensor] = None, into=None):
        """From the forward's inputs and result and the gradient of the result: the
        gradients of q, k and v (into ``into``, three matrices, if given).  saved: that
        forward's ``self.saved``, if another forward has run since."""
        x, bf, dev = self._qkv(q, k, v), torch.bfloat16, q.device
        saved = self.saved if saved is None else saved
        if saved is None or saved.numel() < self.saved_size:
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "backward needs a forward with train=True")
        dx = tuple(torch.empty((self.rows, n), dtype=bf, device=dev)
                   for n in (self.nq, self.nk, self.nk)) if into is None else into
        if self.ws is None:
            self.ws = torch.empty(pf_window_attn_workspace_size(self.desc), dtype=torch.uint8,
                                  device=dev)
        s = self.bwd(self.ref, byref(x), out.data_ptr(), _rows("out", out, self.rows, self.nq, bf),
                     saved.data_ptr(), dout.data_ptr(), _rows("dout", dout, self.rows, self.nq, bf),
                     byref(self._qkv(*dx)), self.ws.data_ptr(), self.ws.numel(), _stream(q))
        if s:
            _check(s)
        return dx


class PagedKVCache:
    """Keys and values of ``batch`` sequences of one layer in a pool of pages.

    ``table`` and ``len`` (device tensors) may be shared by the caches of all
    layers: pass those of the first.  A step: ``reserve`` pages for the new rows
    (host), ``advance`` the lengths once, then ``append`` and ``attend`` layer by
    layer.  ``rope`` (a QKRope) is applied to keys, and queries, on the way in;
    without it they are taken as they are."""

    def __init__(self, batch: int, n_heads: int, n_kv: int, dh: int, page: int, n_pages: int,
                 max_pages: int, rope: Optional[QKRope] = None, window: int = 0, n_sink: int = 0,
                 K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None,
                 table: Optional[torch.Tensor] = None, len: Optional[torch.Tensor] = None,
                 device="cuda"):
        self.batch, self.n_heads, self.n_kv, self.dh, self.page = batch, n_heads, n_kv, dh, page
        self.n_pages, self.max_pages = n_pages, max_pages
        self.rope = rope or QKRope(n_heads, n_kv, dh, pairs=())
        shape = (n_pages, n_kv, page, dh)
        self.K, self.V = (torch.zeros(shape, dtype=torch.bfloat16, device=device) if t is None else t
                          for t in (K, V))
        for t in (self.K, self.V):
            if tuple(t.shape) != shape or t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ProxyFormerError(PF_ERR_INVALID_ARG, f"K and V must be contiguous bf16 {shape}")
        self.table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device) \
            if table is None else table
        self.len = torch.zeros(batch, dtype=torch.int32, device=device) if len is None else len
        self.nq, self.nk = n_heads * dh, n_kv * dh
        self.desc = PagedDesc(batch, n_heads, n_kv, dh, page, max_pages, n_pages, window, n_sink)
        self.cache = PagedCache(self.K.data_ptr(), self.V.data_ptr(),
                                _ints("table", self.table, batch, max_pages),
                                _ints("len", self.len, batch))
        self.ref, self.cref = byref(self.desc), byref(self.cache)
        self.f_append, self.f_attn = load().pf_paged_append, load().pf_paged_attn
        self.ws = torch.empty(max(16, pf_paged_attn_workspace_size(self.desc)), dtype=torch.uint8,
                              device=device)
        self.free = list(range(n_pages - 1, -1, -1))  # pages that reserve() hands out
        self.held = [[] for _ in range(batch)]        # and has handed out, by sequence

    def reserve(self, rows: Sequence[int]) -> None:
        """Pages for rows[b] rows in all of every sequence b (host bookkeeping; a
        cache that was given its table keeps its own)."""
        need = [max(0, -(-int(r) // self.page) - len(p)) for r, p in zip(rows, self.held)]
        if sum(need) > len(self.free) or any(
                n + len(p) > self.max_pages for n, p in zip(need, self.held)):
            raise ProxyFormerError(PF_ERR_CAPACITY, "no pages left for these rows")
        for b, n in enumerate(need):
            if n:
                new = [self.free.pop() for _ in range(n)]
                at = len(self.held[b])
                self.held[b] += new
                self.table[b, at:at + n] = torch.tensor(new, dtype=torch.int32,
                                                        device=self.table.device)

    def release(self, b: int) -> None:
        """Sequence b gives its pages back and is empty."""
        self.free += self.held[b][::-1]
        self.held[b] = []
        self.len[b] = 0

    def advance(self, start: Optional[torch.Tensor] = None) -> None:
        """The lengths at the start of a step: start[b+1] - start[b] more rows of
        every sequence b, or one."""
        pf_paged_advance(self.desc, _ints("start", start, self.batch + 1), self.cache,
                         _stream(self.len))

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
               start: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """The step's tokens, k, v [rows, n_kv*dh], into the cache; returns their
        queries q [rows, n_heads*dh] normed and turned (None without them).  start
        [batch+1] int32: first token of every sequence; None: one each."""
        rows, bf = k.shape[0], torch.bfloat16
        lk, lv = _rows("k", k, rows, self.nk, bf), _rows("v", v, rows, self.nk, bf)
        if q is None:
            x, out, po, lo = QKV(None, k.data_ptr(), v.data_ptr(), 0, lk, lv), None, None, 0
        else:
            x = QKV(q.data_ptr(), k.data_ptr(), v.data_ptr(), _rows("q", q, rows, self.nq, bf), lk, lv)
            out = torch.empty((rows, self.nq), dtype=bf, device=q.device) if out is None else out
            po, lo = out.data_ptr(), _rows("out", out, rows, self.nq, bf)
        r = self.rope
        s = self.f_append(self.ref, r.ref, rows, byref(x), r.pw_q, r.pw_k,
                          _ints("start", start, self.batch + 1), _ints("pos", pos, rows, r.n_axes),
                          self.cref, po, lo, _stream(k))
        if s:
            _check(s)
        return out

    def attend(self, q: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of every sequence's newest token, q [batch, n_heads*dh]."""
        n, bf = self.batch, torch.bfloat16
        out = torch.empty((n, self.nq), dtype=bf, device=q.device) if out is None else out
        s = self.f_attn(self.ref, q.data_ptr(), _rows("q", q, n, self.nq, bf), self.cref,
                        out.data_ptr(), _rows("out", out, n, self.nq, bf), self.ws.data_ptr(),
                        self.ws.numel(), _stream(q))
        if s:
            _check(s)
        return out
