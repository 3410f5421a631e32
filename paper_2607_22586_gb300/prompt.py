"""Torch-facing conveniences around what comes before a selection: rotary positions of Q and
K rows, and attention over whole prompts. PyTorch only provides device memory and
streams here.

    rotary = Rotary(128, theta=1e6, sections=(16, 24, 24))
    attention = PromptAttention(28, 4, 128, torch.bfloat16, cu_seqlens)
    for layer in range(28):
        q, k = rotary(q, k, positions)            # [T, H, d]
        out = attention(q, k, v)
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional, Sequence

import torch

from . import _lib as L
from .selector import _DT


def _on(device: torch.device):
    return nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _no_gradient(*ts: Optional[torch.Tensor]) -> None:
    """Results carry no gradient, so rows that one is wanted of are refused."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in ts):
        raise ValueError("no gradient is taken here: call it under torch.no_grad(), or with detached rows")


def _token_stride(t: torch.Tensor) -> int:
    """The elements between two tokens of t [..., T, heads, d], whose heads are dense."""
    heads, d = t.shape[-2:]
    if (d > 1 and t.stride(-1) != 1) or (heads > 1 and t.stride(-2) != d) \
            or (t.shape[-3] > 1 and t.stride(-3) < heads * d):
        raise ValueError("a token's heads must be dense, and the tokens without overlap")
    return t.stride(-3) if t.shape[-3] > 1 else heads * d


def _layer_stride(t: torch.Tensor, layers: int) -> int:
    """The elements between two layers of t [L, T, heads, d], 0 for a single one."""
    if layers == 1 or not t.numel():
        return 0
    tokens, row, dense = t.shape[-3], _token_stride(t), t.shape[-2] * t.shape[-1]
    behind = t.stride(0) >= (tokens - 1) * row + dense
    beside = t.stride(0) >= dense and row >= (layers - 1) * t.stride(0) + dense     # in a token's row
    if not behind and not beside:
        raise ValueError("layers must lie one behind another or side by side in a token's row, without overlap")
    return t.stride(0)


class Rotary:
    """Rotation of heads of ``head_dim`` to positions: the first ``rot_dims`` of them (0 = all) in
    pairs (j, j + rot_dims / 2) or, ``interleaved``, (2j, 2j + 1). ``sections``: consecutive pairs
    that turn with each of two or three axes of positions. ``scaling`` and what follows it:
    frequencies of contexts longer than the trained one (rope_frequencies; "parts" blends linearly in a
    pair's turns, and models whose blend is linear in the pair's index want ``inv_freq``), or
    ``inv_freq`` and ``amplitude`` themselves."""

    def __init__(self, head_dim: int, rot_dims: int = 0, theta: float = 10000.0, layout: str = "half",
                 sections: Optional[Sequence[int]] = None, scaling: str = "none", factor: float = 1.0,
                 original_length: float = 0.0, low_turns: float = 1.0, high_turns: float = 32.0,
                 inv_freq: Optional[Sequence[float]] = None, amplitude: Optional[float] = None):
        self.head_dim, self.layout = head_dim, layout
        self.sections = list(sections) if sections is not None else None
        if inv_freq is None:
            inv_freq, own = L.rope_frequencies(rot_dims or head_dim, theta, scaling, factor, original_length,
                                               low_turns, high_turns)
            amplitude = own if amplitude is None else amplitude
        elif rot_dims and rot_dims != 2 * len(inv_freq):
            raise ValueError(f"{len(inv_freq)} frequencies for {rot_dims} rotated dimensions")
        self.inv_freq, self.amplitude = list(inv_freq), 1.0 if amplitude is None else float(amplitude)

    def __call__(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor,
                 in_place: bool = False, inverse: bool = False):
        """q [T, Hq, d] and k [T, Hkv, d], or [L, T, H, d] of layers at the same positions
        (either may be None); positions int32 [T], or [axes, T]. ``inverse`` turns the other
        way, which is also the rotation's gradient; autograd does not take it (rows that require one
        are refused where gradients are recorded)."""
        _no_gradient(q, k)
        ts = [t for t in (q, k) if t is not None]
        if not ts:
            raise ValueError("nothing to rotate")
        first = ts[0]
        for t in ts:
            if t.dtype not in _DT or t.dtype != first.dtype or t.device != first.device or not t.is_cuda \
                    or t.dim() not in (3, 4) or t.dim() != first.dim() or t.shape[-1] != self.head_dim \
                    or t.shape[:-2] != first.shape[:-2]:
                raise ValueError("q and k must be [T, H, d] or [L, T, H, d] of one supported type on one GPU")
        layers, total = (first.shape[0] if first.dim() == 4 else 1), first.shape[-3]
        if positions.device != first.device or positions.shape[-1] != total:
            raise ValueError(f"positions must be [{total}] or [axes, {total}] on the rows' device")
        hq, hkv = (q if q is not None else k).shape[-2], (k if k is not None else q).shape[-2]
        if q is None or hq % hkv:                      # the entry asks for whole groups of heads
            results = [self._rotate(t, None, t.shape[-2], t.shape[-2], layers, total, positions, in_place, inverse)[0]
                       for t in ts]
            return (results[0], results[1]) if len(ts) == 2 else (None, results[0])
        return self._rotate(q, k, hq, hkv, layers, total, positions, in_place, inverse)

    def _rotate(self, q, k, hq, hkv, layers, total, positions, in_place, inverse):
        rotary = L.make_rotary(self.inv_freq, positions, self.layout, self.sections, self.amplitude, inverse)
        shape = L.make_shape(hq, hkv, self.head_dim, 2, _DT[q.dtype], [0, total], [1], n_layers=layers)
        strides = [(_token_stride(t), _layer_stride(t, layers)) if t is not None else (0, 0) for t in (q, k)]
        with _on(q.device):
            outs = [t if t is None or in_place else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k)]
            L.check(L.mmshift_rope(shape, rotary, q, *strides[0], k, *strides[1], *outs, torch.cuda.current_stream()),
                    "mmshift_rope")
        return outs[0], outs[1]


class PromptAttention:
    """Attention over the prompts packed by ``cu_seqlens``, with the workspace of that shape. Calls run
    on the current stream; one is used on one stream at a time."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype,
                 cu_seqlens: Sequence[int], device="cuda"):
        if dtype not in _DT:
            raise ValueError(f"unsupported dtype {dtype}")
        self.dtype, self.device = dtype, torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.total_tokens = int(cu_seqlens[-1])
        self.shape = L.make_shape(n_q_heads, n_kv_heads, head_dim, 2, _DT[dtype], cu_seqlens, [1] * (len(cu_seqlens) - 1))
        self._ws_bytes = L.mmshift_prompt_workspace_size(self.shape)
        self._workspace = torch.zeros(self._ws_bytes, dtype=torch.uint8, device=self.device)

    def __call__(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = True,
                 softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        """q [T, Hq, d], k and v [T, Hkv, d], tokens equally far apart (k and v alike):
        [T, Hq, d]. ``lse`` [T, Hq] float32 receives the log-sum-exp where given. There is no backward
        pass: rows that require a gradient are refused where gradients are recorded."""
        _no_gradient(q, k, v)
        for t, heads in ((q, self.n_q_heads), (k, self.n_kv_heads), (v, self.n_kv_heads)):
            if t.dtype != self.dtype or t.device != self.device or t.shape != (self.total_tokens, heads, self.head_dim):
                raise ValueError(f"rows must be [{self.total_tokens}, {heads}, {self.head_dim}] of {self.dtype} "
                                 f"on {self.device}")
        stride = _token_stride(k)
        if stride != _token_stride(v):
            raise ValueError("k's and v's tokens must be equally far apart")
        with _on(self.device):
            if out is None:
                out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
            elif out.dtype != self.dtype or out.device != self.device or not out.is_contiguous() or out.shape != q.shape:
                raise ValueError("out must be a contiguous tensor like q")
            if lse is not None and (lse.dtype != torch.float32 or lse.device != self.device or not lse.is_contiguous()
                                    or lse.shape != q.shape[:2]):
                raise ValueError("lse must be a contiguous float32 tensor [T, Hq]")
            L.check(L.mmshift_prompt_attention(self.shape, q, _token_stride(q), k, v, stride, causal, softmax_scale, out,
                                               lse, self._workspace, self._ws_bytes, torch.cuda.current_stream()),
                    "mmshift_prompt_attention")
        return out

    def poll(self) -> None:
        """Waits for the current stream and raises what a call reported."""
        with _on(self.device):
            L.check(L.mmshift_poll_status(self._workspace, torch.cuda.current_stream()), "mmshift_poll_status")
