"""Sizes at the ends of 32 bits in the linear layers' calls, refused on the host before any
launch (fake pointers, never dereferenced)."""
import pytest
import torch

from paper_2608_01653_amd import hatq
from test_abi_linear import L, P, cpu_only  # noqa: F401


@cpu_only
@pytest.mark.parametrize("cols", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30 + 1])
def test_combine_columns(L, cols):  # noqa: F811
    for tokens, rows in ((1, 1), (3, 0), (0, 1)):
        assert L.hatq_expert_combine(P, rows, cols, cols, P, P, tokens, 1, P, 0, cols, None) == hatq.HATQ_EUNSUPPORTED


def test_binding_sizes_its_workspace_as_the_library(L):  # noqa: F811
    """The binding forms hatq_linear_ws_bytes' size without the call."""
    x = torch.empty(0)
    for cin, ks in ((1, 64), (64, 64), (65, 128), (192, 192), (4095, 4096), (65536, 65536)):
        w = hatq.LinearWeights(1, cin, 100, 0, 1, ks, 128, P, P, P)
        lin = hatq.PreparedLinear(x, w, 1, cin, 100, ks)
        for rows in (1, 3, 4, 5, 63, 64, 65, 255, 257, 1000):
            assert hatq._linear_ws(lin, rows, None, x).numel() == hatq.hatq_linear_ws_bytes(lin, rows) > 0
        assert hatq._linear_ws(lin, 0, None, x).numel() > 0
