"""A feed-forward block of gated experts on the INT8 linear layers over tokens.

One pass for tokens x, their chosen experts and those experts' weights:
  1. the pairs (token, expert) are sorted by expert (hatq_expert_order);
  2. each token is quantized once and goes through the gated layer of each of its
     experts (hatq_experts_forward: rows gathered from the tokens, silu(g) u in the
     epilogue, float32 hidden rows);
  3. each hidden row is quantized and goes through its expert's second layer
     (hatq_experts_forward, float32 rows: they are summed before the one rounding);
  4. a token's rows are summed with their weights (hatq_expert_combine).

Every step runs in the library's kernels; this module only allocates and sequences
the calls.  With one expert and ids of 0 it is a plain gated feed-forward block.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import hatq


class ExpertMLP:
    def __init__(self, w_in: hatq.PreparedLinear, w_out: hatq.PreparedLinear):
        if not w_in.w.gated or w_out.w.gated:
            raise ValueError("w_in has to be a gated layer and w_out a plain one")
        if w_in.experts != w_out.experts or w_in.cout != w_out.cin:
            raise ValueError(f"w_in gives {w_in.experts} x {w_in.cout} channels, w_out takes "
                             f"{w_out.experts} x {w_out.cin}")
        self.w_in, self.w_out = w_in, w_out

    def __call__(self, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor,
                 out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
        """x [tokens, cin], ids int32 and weights float32 [tokens, topk] -> [tokens, cout]
        of out_dtype (default: x's).  An id outside the experts adds nothing."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self(x, ids, weights, out_dtype)
        ends, src, pos = hatq.hatq_expert_order(ids, self.w_in.experts)
        hidden = hatq.hatq_experts_forward(self.w_in, x, ends, src, out_dtype=torch.float32)
        rows = hatq.hatq_experts_forward(self.w_out, hidden, ends, out_dtype=torch.float32)
        return hatq.hatq_expert_combine(rows, pos, weights, out_dtype=out_dtype or x.dtype)
