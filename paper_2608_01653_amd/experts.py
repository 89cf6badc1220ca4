"""A feed-forward block of gated experts on the INT8 linear layers over tokens.

One pass for tokens x, their chosen experts and those experts' weights (one call of the
library, hatq_expert_mlp):
  1. the pairs (token, expert) are sorted by expert;
  2. each token goes through the gated layer of each of its experts: rows gathered from
     the tokens' codes, silu(g) u in the epilogue, float32 hidden rows;
  3. each hidden row is quantized and goes through its expert's second layer, into
     float32 rows: they are summed before the one rounding;
  4. a token's rows are summed with their weights.

With one expert and ids of 0 it is a plain gated feed-forward block.
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
        return hatq.hatq_expert_mlp(self.w_in, self.w_out, x, ids, weights, out_dtype=out_dtype, stream=stream)
