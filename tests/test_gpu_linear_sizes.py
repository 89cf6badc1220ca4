"""Sizes past 32 bits in the binding of the linear layers: refused, not cut to their low
32 bits (2^32 + 4 tokens are not 4).  The tensors are never read."""
import pytest
import torch

from gpu_util import DEV
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
MANY = 2 ** 32 + 4


def test_sizes_past_32_bits():
    lin = hatq.hatq_pack_linear(torch.zeros((16, 1), dtype=torch.int8, device=DEV), torch.ones(16, device=DEV))
    few_ids = torch.zeros((2, 2), dtype=torch.int32, device=DEV)
    x = torch.empty((MANY, 1), dtype=torch.bfloat16, device=DEV)
    ends = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(4096, dtype=torch.int8, device=DEV)
    y4, s4, q4 = torch.empty((4, 16), device=DEV), torch.empty(4, device=DEV), torch.empty((4, 64), dtype=torch.int8, device=DEV)
    calls = [
        lambda: hatq.hatq_linear_forward(lin, x, y=y4, ws=ws),
        lambda: hatq.hatq_experts_forward(lin, x, ends, y=y4, ws=ws),
        lambda: hatq.hatq_token_quant(x, xq=q4, scale=s4),
        lambda: hatq.hatq_token_quant(x.view(1, MANY), xq=q4, scale=s4),
        lambda: hatq.hatq_token_quant(torch.zeros((4, 64), device=DEV), 2 ** 32 + 64),
        lambda: hatq.hatq_linear_ws_bytes(lin, MANY),
        lambda: hatq.hatq_expert_mlp_ws_bytes(lin, lin, MANY, 1),
        lambda: hatq.hatq_expert_order(few_ids, 2 ** 32 + 4, ends=torch.empty(8, dtype=torch.int32, device=DEV)),
        lambda: hatq.hatq_pack_linear(torch.zeros((16, 64), dtype=torch.int8, device=DEV), torch.ones(16, device=DEV), hblock=2 ** 32 + 64),
    ]
    ids = x.view(torch.int16).view(-1).view(torch.int32).view(-1, 1)[:2 ** 31 + 2]      # (2^31 + 2 ids in the same memory)
    calls += [
        lambda: hatq.hatq_expert_order(ids, 4, ends=torch.empty(4, dtype=torch.int32, device=DEV), src=few_ids, pos=few_ids, ws=ws),
        lambda: hatq.hatq_expert_order(ids.view(1, -1), 4, ends=torch.empty(4, dtype=torch.int32, device=DEV), src=few_ids, pos=few_ids, ws=ws),
        lambda: hatq.hatq_expert_combine(y4, ids, ids.view(torch.float32), y=y4),
    ]
    for i, f in enumerate(calls):
        with pytest.raises(ValueError, match="sizes of at most"):
            f()
            pytest.fail(f"call {i} was taken")
