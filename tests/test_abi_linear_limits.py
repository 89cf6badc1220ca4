"""Sizes at the ends of 32 bits in the linear layers' calls, refused on the host before any
launch (fake pointers, never dereferenced)."""
import pytest

from paper_2608_01653_amd import hatq
from test_abi_linear import L, P, cpu_only  # noqa: F401


@cpu_only
@pytest.mark.parametrize("cols", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30 + 1])
def test_combine_columns(L, cols):  # noqa: F811
    for tokens, rows in ((1, 1), (3, 0), (0, 1)):
        assert L.hatq_expert_combine(P, rows, cols, cols, P, P, tokens, 1, P, 0, cols, None) == hatq.HATQ_EUNSUPPORTED
