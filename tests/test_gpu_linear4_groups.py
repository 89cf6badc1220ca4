"""Linear layers of 4-bit weights in waves that take two groups of 16 channels, at both sizes of a
scale's group, and one group past the last whole set; the reference and its bound are
test_gpu_linear4's, in numpy on the CPU."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, Guarded
from paper_2608_01653_amd import hatq
from test_gpu_linear4 import compare, layer, packed, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cin,cout,dtype", [(17, 2176, 16 * 513 - 3, torch.float32), (32, 2304, 16 * 513, torch.bfloat16),
                                                 (33, 2200, 16 * 515 - 15, torch.float16), (70, 2176, 16 * 257 - 1, torch.bfloat16),
                                                 (129, 2056, 16 * 173 + 5, torch.float32), (100, 1104, 16 * 1025 - 3, torch.float32)])
def test_two_groups_a_wave(rows, cin, cout, dtype, gated, group):
    # (plain layers: at least 256 sets of two groups times tiles of 16, 32 or 64 rows)
    tile = 32 if rows <= 32 else 64
    assert -(-cout // 32) * -(-rows // tile) >= 256 and hatq.load() is not None
    rng = np.random.default_rng(rows + cin)
    codes, scale, bias = layer(rng, cout * (2 if gated else 1), cin, group, True)
    x = tokens(rng, rows, cin, dtype)
    lin = packed(codes, scale, bias, 8, gated)
    assert lin.group == group
    n = hatq.hatq_linear4_ws_bytes(lin, rows)
    assert n > 0
    ws, y = Guarded((n,), torch.int8), Guarded((rows, cout), dtype)
    hatq.hatq_linear4_forward(lin, x.to(DEV), y=y.view, ws=ws.view)
    ws.check("workspace")
    y.check()
    compare(x, y.view, codes, scale, bias, 8, group, gated)
