"""Torch-facing convenience around the paged cache's entry points: owns the pages,
their table and the lengths of a batch's sequences, and a workspace that does for
every call. PyTorch only provides device memory and streams here.

    cache = PagedKVCache(28, 4, 128, torch.bfloat16, batch=1, rows=2048 + 512,
                         n_layers=28, cache_dtype=torch.int8)
    cache.fill(selector, K, V)               # after selector(K, V, qwin)
    for k, v, q in steps:                    # [L, T, H, d] of the step's new tokens
        cache.advance(new)                   # new[b]: tokens of request b
        cache.append(k, v, new)
        for layer in range(28):
            out = cache.attend(q[layer], new, layer)
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional, Sequence, Union

import torch

from . import _lib as L
from .selector import _DT, KVSelector


_KEPT = 256   # combinations of row counts whose shapes are kept


class PagedKVCache:
    """Sequences of ``rows`` rows at most (an int, or one for each layer, request
    and KV head: [L, B, Hkv]), each with its pages from the start. Rows appended to a full
    sequence are left out, and poll() reports it (``capacity``: rows that every sequence
    holds). Calls run on the current stream; a cache is used on one stream at a time."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, batch: int,
                 rows: Union[int, Sequence, torch.Tensor], n_layers: int = 1, page_size: int = 64,
                 cache_dtype: Optional[torch.dtype] = None, device="cuda"):
        cache_dtype = dtype if cache_dtype is None else cache_dtype
        if dtype not in _DT or cache_dtype not in (dtype, torch.int8):
            raise ValueError(f"unsupported dtypes {dtype} with a cache of {cache_dtype}")
        self.dtype, self.cache_dtype = dtype, cache_dtype
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.n_layers, self.batch = n_layers, batch
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        need = torch.as_tensor(rows, dtype=torch.int64).cpu().expand(n_layers, batch, n_kv_heads)
        if int(need.min()) < 1:
            raise ValueError("every sequence needs room for a row")
        pages = (need + page_size - 1) // page_size
        ends = pages.flatten().cumsum(0).view(pages.shape)
        total, most = int(ends.flatten()[-1]), int(pages.max())
        # a sequence's pages follow one another; entries behind them are no pages
        entry = torch.arange(most).expand(*pages.shape, most)
        table = torch.where(entry < pages[..., None], entry + (ends - pages)[..., None], -1)
        self.page_table = table.to(torch.int32).to(self.device)
        self.capacity = (pages * page_size).amin().item()
        self.lens = torch.zeros(pages.shape, dtype=torch.int32, device=self.device)
        make = lambda *s, dt: torch.zeros(s, dtype=dt, device=self.device)  # noqa: E731
        self.k_pages, self.v_pages = (make(total, page_size, head_dim, dt=cache_dtype) for _ in range(2))
        self.k_scales = self.v_scales = None
        if cache_dtype == torch.int8:
            self.k_scales, self.v_scales = (make(total, page_size, dt=torch.float32) for _ in range(2))
        self._all = self._struct(self.page_table, self.lens)
        self._layers = [self._struct(self.page_table[i], self.lens[i]) for i in range(n_layers)]
        self._calls, self._counts, self._captured = {}, {}, []
        # The largest call's: the plans' tiles are full from 256 rows of a KV head on, those
        # of few rows from 17 to 32.
        r = n_q_heads // max(n_kv_heads, 1) or 1
        self._ws_bytes = sum(self._shape([n] * batch, 1)[1] for n in (256, max(32 // r, 1)))
        self._workspace = make(self._ws_bytes, dt=torch.uint8)

    def _struct(self, table, lens):
        return L.make_cache(self.k_pages, self.v_pages, table, lens, self.k_scales, self.v_scales)

    def _shape(self, new: Sequence[int], layers: int):
        """Shape of a call with these numbers of rows, and the workspace that attention needs for it."""
        cu = [0]
        for n in new:
            cu.append(cu[-1] + int(n))
        shape = L.make_shape(self.n_q_heads, self.n_kv_heads, self.head_dim, 2, _DT[self.dtype], cu, [1] * self.batch,
                             n_layers=layers, layer_stride_kv=cu[-1] * self.n_kv_heads * self.head_dim)
        return shape, L.mmshift_cache_workspace_size(shape, self._all), cu[-1]

    def _call(self, new: Sequence[int], layers: int):
        """Shape and rows of calls with these numbers of rows."""
        key = (tuple(new), layers)
        if key not in self._calls:
            if len(new) != self.batch:
                raise ValueError(f"{len(new)} row counts for {self.batch} requests")
            if len(self._calls) >= _KEPT:
                self._calls.clear()
            shape, _, total = self._shape(new, layers)
            self._calls[key] = (shape, total)
        return self._calls[key]

    def _on_device(self):
        return nullcontext() if self.device.index == torch.cuda.current_device() else torch.cuda.device(self.device)

    def _check(self, total: int, heads: int, *ts: torch.Tensor) -> int:
        """The elements between two tokens of ``ts`` [..., T, heads, d]."""
        stride = None
        for t in ts:
            if t.dtype != self.dtype or t.device != self.device or t.shape[-3:] != (total, heads, self.head_dim):
                raise ValueError(f"rows must be [..., {total}, {heads}, {self.head_dim}] of {self.dtype} on {self.device}")
            if t.stride(-1) != 1 or (heads > 1 and t.stride(-2) != self.head_dim) \
                    or (total > 1 and (t.stride(-3) != ts[0].stride(-3) or t.stride(-3) < heads * self.head_dim)):
                raise ValueError("a token's heads must be dense, and the tokens equally far apart, without overlap")
            stride = t.stride(-3)
        return stride if total > 1 else heads * self.head_dim

    def fill(self, selector: KVSelector, K: torch.Tensor, V: torch.Tensor,
             idx: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None) -> None:
        """Starts the sequences with the rows that a selection kept (default: the
        selector's last one): K, V [L, T, Hkv, d] as the selector took them; the first
        ``counts`` [L, B, Hkv] int32 rows of each head's where given."""
        selector._check(K, V)
        if (selector.n_layers, len(selector.budgets), selector.n_kv_heads, selector.head_dim, selector.dtype,
                selector.device) != (self.n_layers, self.batch, self.n_kv_heads, self.head_dim, self.dtype, self.device):
            raise ValueError("the selector's shape is not the cache's")
        for t, like in ((idx, selector.out_idx.shape), (counts, self.lens.shape)):
            if t is not None and (t.dtype != torch.int32 or t.device != self.device or not t.is_contiguous()
                                  or t.shape != like):
                raise ValueError("idx [L, R, Hkv] and counts [L, B, Hkv] must be contiguous int32 tensors")
        if idx is None:
            idx, counts = selector.out_idx, selector.kept_count if counts is None else counts
        with self._on_device():
            L.check(L.mmshift_cache_fill(selector.shape, self._all, K, V, idx, counts, self._workspace, self._ws_bytes,
                                         torch.cuda.current_stream()), "mmshift_cache_fill")

    def advance(self, new: Sequence[int]) -> None:
        """Counts ``new[b]`` rows more in every sequence of request b, for all layers.
        (To be captured, counts that differ have to have been used once before.)"""
        if len(new) != self.batch:
            raise ValueError(f"{len(new)} row counts for {self.batch} requests")
        key = tuple(int(n) for n in new)
        if len(set(key)) == 1:
            self.lens.add_(key[0])
            return
        if key not in self._counts:
            if len(self._counts) >= _KEPT:
                self._counts.clear()
            self._counts[key] = torch.tensor(key, dtype=torch.int32, device=self.device)[None, :, None]
        counts = self._counts[key]
        if self.lens.is_cuda:
            with self._on_device():                        # whichever is current for the caller
                if torch.cuda.is_current_stream_capturing():
                    self._captured.append(counts)          # read by every replay
                else:                                      # may be dropped while another stream than its own reads it
                    counts.record_stream(torch.cuda.current_stream())
        self.lens.add_(counts)

    def append(self, K: torch.Tensor, V: torch.Tensor, new: Sequence[int], layer: Optional[int] = None) -> None:
        """The new tokens' rows (counted by advance() before): K, V [L, T, Hkv, d], or
        [T, Hkv, d] of one layer."""
        layers = self.n_layers if layer is None else 1
        shape, total = self._call(new, layers)
        stride = self._check(total, self.n_kv_heads, K, V)
        if layer is not None and (K.dim() != 3 or V.dim() != 3):
            raise ValueError("rows of one layer must be [T, Hkv, d]")
        if layer is None and (K.dim() != 4 or V.dim() != 4 or len(K) != layers or len(V) != layers
                              or (layers > 1 and K.stride(0) != V.stride(0))):
            raise ValueError("rows of all layers must be [L, T, Hkv, d], K's and V's laid out alike")
        shape.layer_stride_kv = K.stride(0) if layer is None else 0
        with self._on_device():
            L.check(L.mmshift_cache_append(shape, self._all if layer is None else self._layers[layer], K, V, stride,
                                           self._workspace, self._ws_bytes, torch.cuda.current_stream()), "mmshift_cache_append")

    def attend(self, q: torch.Tensor, new: Sequence[int], layer: int = 0, causal: bool = True,
               softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        """Attention of the new tokens' queries q [T, Hq, d] over a layer's sequences:
        [T, Hq, d]. ``lse`` [T, Hq] float32 receives the log-sum-exp where given."""
        shape, total = self._call(new, 1)
        stride = self._check(total, self.n_q_heads, q)
        if q.dim() != 3:
            raise ValueError("queries must be [T, Hq, d]")
        with self._on_device():
            if out is None:
                out = torch.empty((total, self.n_q_heads, self.head_dim), dtype=self.dtype, device=self.device)
            elif out.dtype != self.dtype or out.device != self.device or not out.is_contiguous() or out.shape != q.shape:
                raise ValueError("out must be a contiguous tensor like q")
            if lse is not None and (lse.dtype != torch.float32 or lse.device != self.device or not lse.is_contiguous()
                                    or lse.shape != q.shape[:2]):
                raise ValueError("lse must be a contiguous float32 tensor [T, Hq]")
            L.check(L.mmshift_cache_attention(shape, self._layers[layer], q, stride, causal, softmax_scale, out, lse,
                                              self._workspace, self._ws_bytes, torch.cuda.current_stream()), "mmshift_cache_attention")
        return out

    def read(self, rows: Sequence[int], first: Optional[torch.Tensor] = None):
        """The first ``rows[b]`` rows of each sequence of request b (from ``first``
        [L, B, Hkv] int32 on, where given), zeros behind a sequence's end: K and V
        [L, T, Hkv, d]."""
        shape, total = self._call(rows, self.n_layers)
        if first is not None and (first.dtype != torch.int32 or first.device != self.device
                                  or not first.is_contiguous() or first.shape != self.lens.shape):
            raise ValueError("first must be a contiguous int32 tensor [L, B, Hkv]")
        with self._on_device():
            k, v = (torch.empty((self.n_layers, total, self.n_kv_heads, self.head_dim), dtype=self.dtype,
                                device=self.device) for _ in range(2))
            L.check(L.mmshift_cache_read(shape, self._all, first, k, v, self._workspace, self._ws_bytes,
                                         torch.cuda.current_stream()), "mmshift_cache_read")
        return k, v

    def poll(self) -> None:
        """Waits for the current stream and raises what a call on the cache reported."""
        with self._on_device():
            L.check(L.mmshift_poll_status(self._workspace, torch.cuda.current_stream()), "mmshift_poll_status")
