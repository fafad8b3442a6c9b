"""Attention of the local stream (PyTorch holds memory).

``QKRope`` norms and rotates queries and keys (``pf_qk_rope_*``), ``WindowAttention``
is causal attention in a sliding window with sinks (``pf_window_attn_*``) and
``PagedKVCache`` keeps the keys and values of many sequences in pages
(``pf_paged_*``), in bf16 or quantised to 8 bits: ``append`` writes new tokens' rows,
``attend`` is the attention of every sequence's newest token, or tokens, and ``read``
gives rows back.  All calls run on the current CUDA stream;
none does arithmetic of its own.  An object's calls share its workspace: use it on
one stream at a time.  Matrices are 2D tensors whose rows may lie
apart (a slice of a projection's output serves as it is).
"""
from __future__ import annotations

from ctypes import addressof
from typing import Optional, Sequence, Tuple

import torch

from . import (PF_BF16, PF_ERR_CAPACITY, PF_ERR_CUDA, PF_ERR_INVALID_ARG, PF_F32, PagedCache,
               PagedDesc, PagedExp, ProxyFormerError, QKDesc, WindowDesc, load, pf_paged_advance,
               pf_paged_attn_q8_workspace_size, pf_paged_attn_workspace_size, pf_qk_rope_workspace_size, pf_window_attn_saved_size,
               pf_window_attn_workspace_size)
from .buildlib import binding_tag

load()
try:
    from . import _local
    if getattr(_local, "built_for", None) != binding_tag():
        raise ImportError(f"_local.so was built for {getattr(_local, 'built_for', 'another')}")
except ImportError as e:
    raise ProxyFormerError(PF_ERR_CUDA, "_local.so is not built for this interpreter and torch; run "
                           "`python -m paper_2608_23463_gb300.buildlib`") from e
_local.init(ProxyFormerError)


def _workspace(ws: Optional[torch.Tensor], size, desc, q) -> Optional[torch.Tensor]:
    """ws, or a new one of size(desc) bytes where it is not on q's GPU.  (What is no tensor on
    a GPU has none: the call refuses it.)"""
    if not isinstance(q, torch.Tensor) or not q.is_cuda or (ws is not None and ws.device == q.device):
        return ws
    return torch.empty(size(desc), dtype=torch.uint8, device=q.device)


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
        self.desc = QKDesc(n_heads, n_kv, dh, PF_F32 if dtype == torch.float32 else PF_BF16,
                           len(pairs), (pairs + (0, 0, 0))[:3], theta, eps)
        self.at = addressof(self.desc)
        self.ws: Optional[torch.Tensor] = None

    def forward(self, q: torch.Tensor, k: torch.Tensor, L: Optional[int] = None,
                pos: Optional[torch.Tensor] = None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """q [rows, n_heads*dh], k [rows, n_kv*dh] -> the same normed and turned (into
        ``out``, a pair, which may be (q, k) itself).  Positions: pos [rows, axes]
        int32, or the row's place in its sequence of L rows (default: one sequence)."""
        oq, ok = (None, None) if out is None else out
        return _local.rope_fwd(self.at, q, k, L, self.w_q, self.w_k, pos, oq, ok)

    def backward(self, q: torch.Tensor, k: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                 L: Optional[int] = None, pos: Optional[torch.Tensor] = None, out=None):
        """From the forward's inputs and the gradients of its results: the gradients
        of q and k (into ``out``, which may be (dq, dk) itself) and of w_q and w_k
        (None without them)."""
        if self.w_q is not None or self.w_k is not None:
            self.ws = _workspace(self.ws, pf_qk_rope_workspace_size, self.desc, q)
        oq, ok = (None, None) if out is None else out
        return _local.rope_bwd(self.at, q, k, dq, dk, L, self.w_q, self.w_k, pos, oq, ok, self.ws)


class WindowAttention:
    """Causal attention of ``batch`` sequences of L rows: row i sees the last ``window``
    rows up to itself (0: all) and the first ``n_sink``.  bf16, head width 64.  What a row
    does not see does not matter to its result; the backward's inputs must be finite."""

    def __init__(self, batch: int, L: int, n_heads: int, n_kv: int, dh: int = 64, window: int = 0,
                 n_sink: int = 0):
        self.desc = WindowDesc(batch, L, n_heads, n_kv, dh, window, n_sink)
        self.at = addressof(self.desc)
        self.saved_size = pf_window_attn_saved_size(self.desc)
        self.saved: Optional[torch.Tensor] = None  # of the last forward for training
        self.ws: Optional[torch.Tensor] = None

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, train: bool = True,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q [batch*L, n_heads*dh], k, v [batch*L, n_kv*dh] -> [batch*L, n_heads*dh];
        ``train`` keeps what the backward needs beside them."""
        # (saved is a new buffer: the last forward's may still be read on another stream, for
        # which its memory waits)
        out, saved = _local.window_fwd(self.at, q, k, v, out, self.saved_size if train else 0)
        if train:
            self.saved = saved
        return out

    def backward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                 dout: torch.Tensor, saved: Optional[torch.Tensor] = None, into=None):
        """From the forward's inputs and result and the gradient of the result: the
        gradients of q, k and v (into ``into``, three matrices, if given).  saved: that
        forward's ``self.saved``, if another forward has run since."""
        self.ws = _workspace(self.ws, pf_window_attn_workspace_size, self.desc, q)
        dq, dk, dv = (None, None, None) if into is None else into
        return _local.window_bwd(self.at, q, k, v, out, dout, self.saved if saved is None else saved,
                                 dq, dk, dv, self.ws)


class PagedKVCache:
    """Keys and values of ``batch`` sequences of one layer in a pool of pages.

    ``table`` and ``len`` (device tensors) may be shared by the caches of all
    layers: pass those of the first.  A step: ``reserve`` pages for the new rows
    (host), ``advance`` the lengths once, then ``append`` and ``attend`` layer by
    layer.  ``rope`` (a QKRope) is applied to keys, and queries, on the way in;
    without it they are taken as they are.

    ``dtype`` torch.int8 holds each row (one token and key head) as whole numbers
    K, V and an exponent K_exp, V_exp [n_pages, n_kv, page] of its own, x * 2^e with
    the least e that the row allows: half the memory, each value off by at most
    1/127 of its row's largest.  All operators take such a cache."""

    def __init__(self, batch: int, n_heads: int, n_kv: int, dh: int, page: int, n_pages: int,
                 max_pages: int, rope: Optional[QKRope] = None, window: int = 0, n_sink: int = 0,
                 K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None,
                 table: Optional[torch.Tensor] = None, len: Optional[torch.Tensor] = None,
                 device="cuda", dtype: torch.dtype = torch.bfloat16,
                 K_exp: Optional[torch.Tensor] = None, V_exp: Optional[torch.Tensor] = None):
        self.batch, self.n_heads, self.n_kv, self.dh, self.page = batch, n_heads, n_kv, dh, page
        self.n_pages, self.max_pages = n_pages, max_pages
        self.rope = rope or QKRope(n_heads, n_kv, dh, pairs=())
        if dtype not in (torch.bfloat16, torch.int8):
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "dtype must be torch.bfloat16 or torch.int8")
        self.dtype = dtype
        shape = (n_pages, n_kv, page, dh)
        self.K, self.V = (torch.zeros(shape, dtype=dtype, device=device) if t is None else t
                          for t in (K, V))
        for t in (self.K, self.V):
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
                raise ProxyFormerError(PF_ERR_INVALID_ARG, f"K and V must be contiguous {dtype} {shape}")
        self.K_exp, self.V_exp = K_exp, V_exp
        if dtype == torch.int8:
            self.K_exp, self.V_exp = (torch.zeros(shape[:3], dtype=torch.int8, device=device) if t is None else t
                                      for t in (K_exp, V_exp))
        for t in (self.K_exp, self.V_exp):
            if (t is None) != (dtype == torch.bfloat16) or t is not None and (
                    tuple(t.shape) != shape[:3] or t.dtype != torch.int8 or not t.is_contiguous()):
                raise ProxyFormerError(PF_ERR_INVALID_ARG, f"K_exp and V_exp are an int8 cache's, contiguous int8 {shape[:3]}")
        self.table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device) \
            if table is None else table
        self.len = torch.zeros(batch, dtype=torch.int32, device=device) if len is None else len
        for name, t, shape in (("table", self.table, (batch, max_pages)), ("len", self.len, (batch,))):
            if tuple(t.shape) != shape or t.dtype != torch.int32 or not t.is_contiguous():
                raise ProxyFormerError(PF_ERR_INVALID_ARG, f"{name} must be contiguous int32 {shape}")
        if not all(t.is_cuda and t.device == self.K.device for t in (self.V, self.table, self.len, self.K_exp, self.V_exp)
                   if t is not None):
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "K, V, table and len must be on one GPU")
        self.desc = PagedDesc(batch, n_heads, n_kv, dh, page, max_pages, n_pages, window, n_sink)
        self.cache = PagedCache(self.K.data_ptr(), self.V.data_ptr(),
                                self.table.data_ptr(), self.len.data_ptr())
        self.at, self.at_cache, self.at_exp = addressof(self.desc), addressof(self.cache), 0
        if dtype == torch.int8:
            self.exp = PagedExp(self.K_exp.data_ptr(), self.V_exp.data_ptr())
            self.at_exp = addressof(self.exp)
        size = pf_paged_attn_workspace_size if dtype == torch.bfloat16 else pf_paged_attn_q8_workspace_size
        self.ws = torch.empty(max(16, size(self.desc)), dtype=torch.uint8, device=self.K.device)
        self.free = list(range(n_pages - 1, -1, -1))  # pages that reserve() hands out
        self.held = [[] for _ in range(batch)]        # and has handed out, by sequence
        self.left = set()                             # sequences released and not begun again

    def reserve(self, rows: Sequence[int]) -> None:
        """Pages for rows[b] rows in all of every sequence b (host bookkeeping; a
        cache that was given its table keeps its own).  A released sequence that gets
        pages again begins empty."""
        need = [max(0, -(-int(r) // self.page) - len(p)) for r, p in zip(rows, self.held)]
        if sum(need) > len(self.free) or any(
                n + len(p) > self.max_pages for n, p in zip(need, self.held)):
            raise ProxyFormerError(PF_ERR_CAPACITY, "no pages left for these rows")
        for b, n in enumerate(need):
            if n:
                if b in self.left:  # steps of one token have counted its rows on
                    self.left.remove(b)
                    self.len[b] = 0
                new = [self.free.pop() for _ in range(n)]
                at = len(self.held[b])
                self.held[b] += new
                self.table[b, at:at + n] = torch.tensor(new, dtype=torch.int32,
                                                        device=self.table.device)

    def release(self, b: int) -> None:
        """Sequence b gives its pages back and is empty.  Its place in the table is cleared:
        another sequence may own the pages when a step of one token for every sequence
        reaches b too, which is flagged (PF_ERR_CAPACITY) and writes nothing."""
        self.table[b, :len(self.held[b])] = -1
        self.free += self.held[b][::-1]
        self.held[b] = []
        self.left.add(b % self.batch)
        self.len[b] = 0

    def advance(self, start: Optional[torch.Tensor] = None) -> None:
        """The lengths at the start of a step: start[b+1] - start[b] more rows of
        every sequence b, or one."""
        if start is not None and (not isinstance(start, torch.Tensor) or start.device != self.len.device
                                  or tuple(start.shape) != (self.batch + 1,)
                                  or start.dtype != torch.int32 or not start.is_contiguous()):
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "start must be batch + 1 int32 values on the cache's GPU")
        with torch.cuda.device(self.len.device):
            pf_paged_advance(self.desc, start, self.cache, torch.cuda.current_stream().cuda_stream)

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
               start: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """The step's tokens, k, v [rows, n_kv*dh], into the cache; returns their
        queries q [rows, n_heads*dh] normed and turned (None without them).  start
        [batch+1] int32: first token of every sequence; None: one each."""
        r = self.rope
        return _local.paged_append(self.at, r.at, self.at_cache, self.at_exp, self.len, q, k, v, r.w_q, r.w_k,
                                   start, pos, out)

    def attend(self, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               start: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of every sequence's newest token, q [batch, n_heads*dh], or with start
        (as in append) of the step's tokens, q [rows, n_heads*dh]: each sees the rows up to
        its own.  Rows of q from start[batch] on are left alone in out."""
        if start is not None:
            return _local.paged_chunk(self.at, self.at_cache, self.at_exp, self.len, q, start, out)
        return _local.paged_attn(self.at, self.at_cache, self.at_exp, self.len, q, out, self.ws)

    def read(self, start: Optional[torch.Tensor] = None, rows: Optional[int] = None,
             out=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The last rows of every sequence, start[b+1] - start[b] of them (None: one), as they
        lie in the cache: keys (normed and turned) and values, [rows, n_kv*dh] bf16 (into ``out``,
        a pair).  rows: start[batch], or more: what is past it is left alone."""
        if rows is None and out is not None:
            rows = out[0].shape[0]
        if rows is None and start is not None:
            raise ProxyFormerError(PF_ERR_INVALID_ARG, "read needs the number of rows beside start")
        k, v = (None, None) if out is None else out
        return _local.paged_read(self.at, self.at_cache, self.at_exp, self.len,
                                 self.batch if rows is None else rows, start, k, v)
