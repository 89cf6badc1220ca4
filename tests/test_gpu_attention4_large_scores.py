"""Attention over the 4-bit cache with scores so large that float32 does not resolve a softmax of
them: a result is still a mean of the values of positions that the scores' rounding leaves at the
top, mostly of one, and neither NaN nor 0.

Positions (u = 2^-24): a computed score is within e = (80 u + 2^-22, or 2^-11 for bfloat16 rows in one
half) sum |q k| of its own, as in cache4_util.attention64, and the unit of the weights is within 4 steps
of a score, 2^-21 of it; what is taken down to 2^15 units is so by its weight times its scale, and a
position's scales are within 2^8 of another's here.  So one that lies 2 e + 2^-20 |top| + ln 2^8 + 25 below
the top has at most exp(-25) of its weight.  Result: between the least and the largest of the others'
values, but for the weights' rounding (2^-11, in two halves 2^-21), the sums' (count + 64) u and the
left out positions' count exp(-25), all of them of the values' magnitudes."""
import numpy as np
import pytest
import torch

from cache4_util import ROUND, U, Sequences, butterfly, butterfly_abs, held
from gpu_util import DEV, dev
from paper_2608_01653_amd import hatq
from test_gpu_attention4 import queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def check(s, i, q, y, first, fine, scale=None):
    """Rows q, y of sequence i, the first of them at position `first`."""
    k, v = (held(x, s.hblock) for x in s.of(i))
    scale = s.dim ** -0.5 if scale is None else scale
    share, one = q.shape[1] // s.heads, 0
    q, got, (rel, low) = q.float().numpy().astype(np.float64), y.double().cpu().numpy(), ROUND[y.dtype]
    for row in range(len(q)):
        n = min(first + row + 1, len(k))
        for h in range(q.shape[1]):
            kk, vv, qt = k[:n, h // share], v[:n, h // share], butterfly(q[row, h], s.hblock)
            score, size = kk @ qt * (scale / s.hblock), np.abs(kk) @ np.abs(qt) * (scale / s.hblock)
            e = (80 * U + (2.0 ** -22 if fine else 2.0 ** -11)) * size.max()
            top = score > score.max() - (2 * e + 2.0 ** -20 * np.abs(score).max() + 8 * np.log(2.0) + 25)
            one += top.sum() == 1
            of = butterfly(vv[top], s.hblock) / s.hblock
            off = (2.0 ** -21 if fine else 2.0 ** -11) + (n + 64) * U + n * np.exp(-25.0)
            off = off * butterfly_abs(np.abs(vv).max(0)[None], s.hblock)[0]
            off = off + rel * np.abs(got[row, h]) + low
            assert (got[row, h] >= of.min(0) - off).all() and (got[row, h] <= of.max(0) + off).all(), (row, h, top.sum(), score.max())
    return one


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power", [16, 20, 22, 24, 26, 28, 31, 40, 80])
@pytest.mark.parametrize("dim,hblock,page", [(64, 64, 16), (128, 128, 64), (192, 64, 64), (256, 128, 16), (128, 1, 16)])
def test_one_token(dim, hblock, page, power, dtype):
    s = Sequences([1500, 700, 33], 2, dim, hblock, page, dtype, seed=dim + power)
    s.write()
    q = queries(s, [1] * 3, 8, dtype, 2.0 ** power)
    many = 0
    for max_len in (0, 1):      # parts or whole, many waves or one
        y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, max_len=max_len)
        for i, n in enumerate(s.lens_np):
            many += check(s, i, q[i:i + 1], y[i:i + 1], n - 1, dtype != torch.bfloat16)
    # (in two halves, mostly one position is the top)
    assert dtype == torch.bfloat16 or many > 30


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power", [20, 24, 28, 34, 90])
@pytest.mark.parametrize("dim,hblock,page", [(64, 64, 64), (128, 64, 16), (192, 64, 16), (80, 16, 64)])
def test_many_rows(dim, hblock, page, power, dtype):
    """Blocks of many columns, rows small and large among them."""
    new = [130, 7, 370, 1]
    s = Sequences([130, 60, 400, 65], 8, dim, hblock, page, dtype, seed=dim + power)
    s.write()
    q = queries(s, new, 64, dtype)
    q[::3] *= 2.0 ** power
    q[1::3] *= 2.0 ** 10
    ends = np.cumsum(new)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, ends=dev(ends.astype(np.int32)))
    assert not bool(torch.isnan(y).any())
    for i, row in ((0, 0), (0, 1), (0, 129), (1, 133), (2, 200), (2, 300), (2, 506), (3, 507)):
        n = s.lens_np[i] - (ends[i] - row)
        check(s, i, q[row:row + 1, ::8], y[row:row + 1, ::8], n, dtype != torch.bfloat16)


def test_far_below_zero():
    """All scores far below zero, or on both sides of it by turns."""
    for sign in (-1.0, 1.0):
        s = Sequences([900], 1, 64, 64, 64, torch.float32, seed=3)
        s.k = s.k.abs()
        s.k[::2] *= sign
        s.write()
        q = -torch.from_numpy(s.rng.uniform(0.5, 1.0, size=(1, 4, 64)).astype(np.float32)) * 2.0 ** 27
        y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)
        assert check(s, 0, q, y, 899, True) > 0
