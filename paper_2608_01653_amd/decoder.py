"""The two halves of a decoder layer on the library's quantized operators.

CachedAttention  one pass for new tokens' rows x:
  1. the query-key-value layer (INT8 or 4-bit weights);
  2. the new keys and values into the 4-bit cache;
  3. attention of the queries over it;
  4. the output layer.
GatedMLP  the gated layer silu(g) u and the layer after it.

Either takes layers of hatq_prepare_linear / hatq_pack_linear (one expert) or of
hatq_prepare_linear4 / hatq_pack_linear4.  Norms, residuals and positions are the model's.
"""
from __future__ import annotations

from typing import Callable, Optional, Tuple, Union

import torch

from . import hatq

Layer = Union[hatq.PreparedLinear, hatq.PreparedLinear4]


def forward(lin: Layer, x: torch.Tensor, out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """Tokens x through a linear layer of either kind."""
    call = hatq.hatq_linear4_forward if isinstance(lin, hatq.PreparedLinear4) else hatq.hatq_linear_forward
    return call(lin, x, out_dtype, stream=stream)


def _plain(lin: Layer, name: str):
    if getattr(lin, "experts", 1) != 1:
        raise ValueError(f"{name}: one layer expected, got {lin.experts} experts")
    if lin.w.gated:
        raise ValueError(f"{name}: a plain layer expected, got a gated one")


class CachedAttention:
    def __init__(self, w_qkv: Layer, w_out: Layer, cache: hatq.Cache4, q_heads: int, scale: Optional[float] = None):
        """w_qkv gives the queries of q_heads heads, then the cache's heads of keys, then of
        values; w_out takes the heads' results."""
        _plain(w_qkv, "w_qkv")
        _plain(w_out, "w_out")
        if q_heads % cache.heads:
            raise ValueError(f"{q_heads} query heads over {cache.heads} heads of the cache")
        if w_qkv.cout != (q_heads + 2 * cache.heads) * cache.dim or w_out.cin != q_heads * cache.dim:
            raise ValueError(f"w_qkv of {(q_heads + 2 * cache.heads) * cache.dim} channels and w_out of {q_heads * cache.dim} "
                             f"input channels expected, got {w_qkv.cout} and {w_out.cin}")
        self.w_qkv, self.w_out, self.cache, self.q_heads, self.scale = w_qkv, w_out, cache, q_heads, scale

    def __call__(self, x: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, ends: Optional[torch.Tensor] = None,
                 rotate: Optional[Callable[[torch.Tensor, torch.Tensor], Tuple[torch.Tensor, torch.Tensor]]] = None,
                 window: int = 0, max_len: int = 0, stream=None) -> torch.Tensor:
        """x [rows, width], the last tokens of their sequences (lens counts them) -> [rows,
        width].  table, lens, ends, window, max_len: as hatq_attention4; rotate(q, k): what the
        model does to queries and keys before they meet."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self(x, table, lens, ends, rotate, window, max_len)
        cache = self.cache
        qkv = forward(self.w_qkv, x).unflatten(1, (self.q_heads + 2 * cache.heads, cache.dim))
        q, k, v = qkv.split((self.q_heads, cache.heads, cache.heads), dim=1)
        if rotate is not None:
            q, k = rotate(q, k)
        hatq.hatq_cache4_append(cache, k, v, table, lens, ends)
        y = hatq.hatq_attention4(cache, q, table, lens, ends, scale=self.scale, window=window, max_len=max_len)
        return forward(self.w_out, y.flatten(1))


class GatedMLP:
    def __init__(self, w_in: Layer, w_out: Layer):
        if getattr(w_in, "experts", 1) != 1 or not w_in.w.gated:
            raise ValueError("w_in: one gated layer expected")
        _plain(w_out, "w_out")
        if w_in.cout != w_out.cin:
            raise ValueError(f"w_in gives {w_in.cout} channels, w_out takes {w_out.cin}")
        self.w_in, self.w_out = w_in, w_out

    def __call__(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """x [rows, width] -> [rows, w_out's channels]."""
        return forward(self.w_out, forward(self.w_in, x, stream=stream), stream=stream)
