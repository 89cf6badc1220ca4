"""The gated unit g / (1 + exp(-g)) u of the linear layers over tokens against 64 bits,
over every gate that fp32 tells apart from none, in each of the products' kernels.

A layer of zero codes has z = bias, exactly, so the gates are the biases.  Tolerance (u =
2^-24): exp(-g) = 2^n 2^f with f off by at most half an ulp of 1/2 and the hardware's
exponential by 2 u, 3 u together; 1 + exp(-g), the quotient and the product with u round
once each, the quotient's correction to within another u: 7 u, and the tests allow 8 u
|y|, whatever the gate.
"""
import numpy as np
import pytest
import torch

from gpu_util import DEV, dev, host
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def gated_rows(g, u, rows, forward):
    """y [rows, len(g)] of a layer whose gates are g and whose values are u."""
    n = len(g)
    lin = hatq.hatq_pack_linear(torch.zeros((2 * n, 64), dtype=torch.int8, device=DEV), torch.ones(2 * n, device=DEV),
                                dev(np.concatenate((g, u)).astype(np.float32)), gated=True)
    if forward:
        return hatq.hatq_linear_forward(lin, torch.zeros((rows, 64), device=DEV))
    return hatq.hatq_linear_int8(lin, torch.zeros((rows, 64), dtype=torch.int8, device=DEV), torch.ones(rows, device=DEV))


# few rows of floats, of codes, and tiles
@pytest.mark.parametrize("rows,forward", [(1, True), (1, False), (40, False), (300, True), (700, False), (3000, False)])
def test_gated_unit(rows, forward):
    rng = np.random.default_rng(rows)
    g = np.concatenate([np.linspace(-88.5, 88.5, 1500), rng.normal(0, 3, 1500), 10.0 ** rng.uniform(-30, 1, 600),
                        -10.0 ** rng.uniform(-30, 1, 600), [0.0, -0.0, 87.0, -87.0, 86.99999, -86.99999, 1e30, 3e38]]).astype(np.float32)
    rng.shuffle(g)
    u = rng.uniform(-2, 2, len(g)).astype(np.float32)
    y = gated_rows(g, u, rows, forward)
    assert bool((y == y[:1]).all())
    g, u = g.astype(np.float64), u.astype(np.float64)
    ref = g / (1 + np.exp(-np.maximum(g, -700))) * u
    got = host(y[0].double())
    over = np.abs(ref) > float(np.finfo(np.float32).max)      # fp32 holds no such product
    assert np.array_equal(got[over], np.sign(ref[over]) * np.inf)
    off, ref = np.where(over, 0.0, np.abs(got - ref)) / U, np.where(over, 0.0, ref)
    bad = off > 8 * np.abs(ref) + 2.0 ** -120
    assert not bad.any(), [(float(a), float(b)) for a, b in zip(g[bad][:5], (off[bad] / np.abs(ref[bad]))[:5])]


@pytest.mark.parametrize("rows,forward", [(1, True), (40, False), (700, False)])
def test_gated_unit_ends(rows, forward):
    """Gates that are not finite or give nothing, each beside ordinary ones."""
    inf, nan = np.inf, np.nan
    g = np.array([1.0, inf, 2.0, -3.0, 1.0, -200.0, nan, 0.5, -inf, -1e30, 88.0, 0.25], np.float32)
    y = host(gated_rows(g, np.full(len(g), 2.0, np.float32), rows, forward)[rows - 1].double())
    with np.errstate(all="ignore"):
        ref = g.astype(np.float64) / (1 + np.exp(-g.astype(np.float64))) * 2.0
    finite = np.isfinite(g) & (g > -100)
    assert (np.abs(y[finite] - ref[finite]) <= 8 * U * np.abs(ref[finite])).all()
    assert y[1] == inf and np.isnan(y[6]) and np.isnan(y[8])       # (-inf: -inf / inf)
    assert abs(y[5]) < 2.0 ** -120 and abs(y[9]) < 2.0 ** -120
