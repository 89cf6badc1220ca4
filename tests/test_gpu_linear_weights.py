"""Float weights that are not finite: their channel's outputs say so, no other's change."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, dev, host
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("e,held,cin,b,gated", [(1, 40, 128, 1, False), (1, 33, 700, 4, False), (3, 34, 512, 64, True)])
def test_channels_not_finite(dtype, e, held, cin, b, gated):
    rng = np.random.default_rng(held)
    w = torch.from_numpy(rng.normal(0, 0.1, (e, held, cin)).astype(np.float32)).to(dtype).to(DEV)
    good = hatq.hatq_prepare_linear(w, hblock=b, gated=gated)
    bad = w.clone()
    at = [(0, 3, 0, float("nan")), (0, 17, cin - 1, float("inf")), (e - 1, 20, cin // 2, float("-inf")), (e - 1, held - 1, 65, float("nan"))]
    for i, c, d, v in at:
        bad[i, c, d] = v
    lin = hatq.hatq_prepare_linear(bad, hblock=b, gated=gated)
    x = dev(rng.normal(0, 1, (2 * e, cin)).astype(np.float32))
    ends = dev((2 * np.arange(1, e + 1)).astype(np.int32))
    y, ref = (host(hatq.hatq_experts_forward(w_, x, ends)) for w_ in (lin, good))
    nan = np.zeros(y.shape, bool)
    for i, c, _, _ in at:
        nan[2 * i:2 * i + 2, c % lin.cout] = True     # (a gate or a value of that output)
    assert np.array_equal(np.isnan(y), nan)
    assert np.array_equal(y[~nan], ref[~nan])


def test_weights_past_float32():
    """Finite weights whose transform overflows fp32."""
    w = torch.full((2, 64), 3e38, device=DEV)
    w[1] = 1.0
    y = host(hatq.hatq_linear_forward(hatq.hatq_prepare_linear(w, hblock=64), torch.ones((1, 64), device=DEV)))
    assert np.isnan(y[0, 0]) and abs(y[0, 1] - 64.0) < 1e-3
