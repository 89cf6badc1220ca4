"""Heads that the 4-bit cache cannot hold: one value that is not below 2^102 in magnitude after the
transform, and the head is stored as NaN, codes 0 under scales NaN in all of its groups, whatever its
other values are."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, dev
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
LARGE = 2.0 ** 102


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def stored(x, hblock):
    """The bytes of a cache of keys x and values -x [16, heads, dim]."""
    _, heads, dim = x.shape
    cache = hatq.hatq_cache4_init(1, 16, heads, dim, hblock=hblock, device=DEV)
    cache.buf.zero_()
    hatq.hatq_cache4_append(cache, x, -x, dev(np.zeros((1, 1), np.int32)), dev(np.array([16], np.int32)))
    return cache.buf


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,hblock", [(128, 64), (128, 128), (128, 1), (64, 64), (80, 16), (192, 8), (256, 128), (256, 1)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), LARGE, -LARGE, 1e33])
def test_one_value(value, dim, hblock, dtype):
    rng = np.random.default_rng(dim + hblock)
    x = torch.from_numpy(rng.normal(size=(16, 2, dim)).astype(np.float32)).to(dtype).to(DEV)
    nan = x.clone()
    for row, (head, d) in enumerate([(0, 0), (1, dim - 1), (0, dim // 2), (1, min(63, dim - 1)), (0, dim - 16)]):
        x[3 * row, head, d] = value
        nan[3 * row, head] = float("nan")
    got, want = stored(x, hblock), stored(nan, hblock)
    assert torch.equal(got, want)
    # all of them: no value of the head has a code
    x[5], nan[5] = value, float("nan")
    if hblock == 1:
        assert torch.equal(stored(x, 1), stored(nan, 1))
