"""Which calls of the linear layers of 4-bit weights the binding makes without a workspace, on the
CPU: only ones for which the library asks for none, from sizes alone."""
import ctypes

import pytest
import torch

from paper_2608_01653_amd import hatq

P = 0x10000            # aligned to 256, never dereferenced
MOST = 1 << 24


def layer(cin, cout, gated):
    k_stride, pad = -(-cin // 128) * 128, -(-cout // 16) * 16 * (2 if gated else 1)
    w = hatq.Linear4Weights(cin, cout, int(gated), 1, 128, k_stride, pad, P, P, P)
    return hatq.PreparedLinear4(torch.empty(1, dtype=torch.int8), w, cin, cout, 128, k_stride)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("cin", [1, 128, 500, 512, 700, 1024, 1025, 2000, 2048, 2049, 4096, 8192, 16384, 16385, 65536])
def test_rows_without_a_workspace(cin, gated):
    L = hatq.load(build_if_missing=True)
    for cout in (1, 16, 257, 2048, 4096, 4112, 8192, 8193, 32768):
        lin = layer(cin, cout, gated)

        def need(rows):
            return L.hatq_linear4_ws_bytes(ctypes.byref(lin.w), rows)
        # every count of a few rows, then counts around multiples of 16
        few = list(range(1, min(lin.rows, 300) + 1))
        assert not any(need(n) for n in few + [n for k in range(9, 21) for n in ((1 << k) - 1, 1 << k, (1 << k) + 1) if n <= lin.rows])
        assert not lin.rows or need(lin.rows) == 0
        assert lin.rows == MOST or need(lin.rows + 1) > 0
