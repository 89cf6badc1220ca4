"""Attention over the 4-bit cache where weights, or the scales of a head's groups of 64
channels, are far apart: against 64 bits, each channel by what it is itself made of.

Bounds (u = 2^-24), as cache4_util.attention64, but for each position p and channel d: a weight
times a scale, a = w s, is off by `rel` of itself, 2^-11 in one float16 half and 2^-21 in two, or,
where it is subnormal, by half of float16's least step, 2^-25, of a unit.  The largest a of the row's
positions and of all the head's groups is at least 2^12 units, so that is FLOOR = 2^-37 of it.  A
channel's sum is off by these times its codes |c|, by the score's error (80 roundings, and the query's
halves), and by the float32 sums: u for each of the positions, of the magnitudes of that channel alone
and of the weights' sum."""
import numpy as np
import pytest
import torch

from cache4_util import U, Sequences, butterfly, butterfly_abs, check, quantize
from gpu_util import DEV, dev
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
REL = {True: 2.0 ** -21, False: 2.0 ** -11}
FLOOR = 2.0 ** -37
ROWS = 512      # of 8 heads' 8 queries: blocks of many columns


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def row64(q, k, v, hblock, scale, fine):
    """(y, bound) of one query head [dim] that sees all of k, v [len, dim], float32."""
    (ck, sk), (cv, sv) = ([x.astype(np.float64) for x in quantize(x, hblock)] for x in (k, v))
    qt, kk = butterfly(q.astype(np.float64), hblock), ck * sk
    t = kk @ qt * (scale / hblock)
    w = np.exp(t - t.max())
    size = (np.abs(kk) @ np.abs(qt)).max() * scale / hblock
    a = w[:, None] * sv
    score = np.expm1(2 * (80 * U + (2.0 ** -22 if fine else 2.0 ** -11)) * size)
    weight = np.maximum(REL[fine] * a, FLOOR * a.max())
    off = ((weight + (score + (3 * len(k) + 24) * U) * a) * np.abs(cv)).sum(0)
    return butterfly((a * cv).sum(0), hblock) / hblock / w.sum(), butterfly_abs(off[None], hblock)[0] / w.sum()


def compare(s, q, y, scale, fine, rows):
    """The given rows of y, of one sequence that all of them see whole."""
    k, v = s.of(0)
    share = q.shape[1] // s.heads
    for row in rows:
        want = [row64(q[row, h].float().numpy(), k[:, h // share], v[:, h // share], s.hblock, scale, fine) for h in range(q.shape[1])]
        check(y[row].cpu(), np.stack([w[0] for w in want]), np.stack([w[1] for w in want]), f"row {row}")


def run(s, q, fine, out=None, max_len=0):
    """One row of each query head, then many rows alike of eight."""
    s.write()
    scale = s.dim ** -0.5
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, out_dtype=out, max_len=max_len)
    compare(s, q, y, scale, fine, [0])
    share = 8 // (q.shape[1] // s.heads)
    many = q.unflatten(1, (s.heads, -1)).repeat_interleave(share, dim=2).flatten(1, 2).expand(ROWS, -1, -1)
    y = hatq.hatq_attention4(s.cache, many.to(DEV), s.table, s.lens, causal=False, out_dtype=out, max_len=max_len)
    compare(s, many, y, scale, fine, [0])
    assert bool((y == y[:1]).all())


@pytest.mark.parametrize("max_len", [1, 256])       # a block of one wave, and of eight
@pytest.mark.parametrize("dtype,nats", [(torch.bfloat16, 14), (torch.bfloat16, 18), (torch.float16, 16), (torch.float32, 14), (torch.float32, 18),
                                        (torch.float32, 20)])
def test_a_position_far_ahead(dtype, nats, max_len):
    """One position has nearly all the weight and a value of 0 in half of the channels: there the
    others' weights are all that counts."""
    s = Sequences([4000], 8, 64, 1, 64, torch.float32, seed=nats, poison=False)
    s.k *= 0.05
    s.v[0, :, :32], s.v[0, :, 32:] = 1.0, 0.0
    s.k[0] = nats / 4.0         # the score of a query of 0.5: 64 * 0.5 * nats / 4 / 8
    q = torch.full((1, 16, 64), 0.5, dtype=dtype)
    run(s, q, dtype != torch.bfloat16, torch.bfloat16 if dtype == torch.bfloat16 else torch.float32, max_len)


@pytest.mark.parametrize("dtype,apart", [(torch.bfloat16, 12), (torch.bfloat16, 18), (torch.bfloat16, 24), (torch.float32, 12), (torch.float32, 18),
                                         (torch.float32, 24), (torch.float32, 30)])
@pytest.mark.parametrize("dim,hblock", [(128, 64), (128, 1), (256, 32), (192, 64), (80, 16)])
def test_groups_of_a_head_far_apart(dim, hblock, dtype, apart):
    """Each 64 channels' values 2^apart below those before, or 2^apart below all the first (of
    256: apart / 2 twice and a group like the first again)."""
    s = Sequences([300], 8, dim, hblock, 16, dtype, seed=dim + apart)
    down = [0, apart, apart // 2, 0][:-(-dim // 64)]
    for g, by in enumerate(down):
        s.v[..., 64 * g:64 * g + 64] *= 2.0 ** -by
    q = torch.from_numpy(s.rng.normal(size=(1, 16, dim)).astype(np.float32)).to(dtype)
    run(s, q, dtype != torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("apart", [6, 12, 20, 26])
@pytest.mark.parametrize("dim,hblock", [(128, 64), (128, 1), (192, 32), (80, 16)])
def test_queries_and_keys_far_apart(dim, hblock, apart, dtype):
    """A group of 64 channels with small queries and keys as much larger: it counts as the others.  A
    query's value is also off by half of float16's least step where its largest is at least 2^13,
    2^-38 of it, which moves a score by that of the sum of |k|: row64's error of a score, 2 of it a
    weight, is made larger by as much."""
    s = Sequences([300], 8, dim, hblock, 16, torch.float32, seed=dim + apart)
    s.k[..., 64:] *= 2.0 ** apart
    q = torch.from_numpy(s.rng.normal(size=(1, 16, dim)).astype(np.float32))
    q[..., 64:] *= 2.0 ** -apart
    q = q.to(dtype)
    s.write()
    fine = dtype != torch.bfloat16
    many = q.unflatten(1, (8, 2)).repeat_interleave(4, dim=2).flatten(1, 2).expand(ROWS, -1, -1)
    k, v = s.of(0)
    for rows in (q, many):
        y = hatq.hatq_attention4(s.cache, rows.to(DEV), s.table, s.lens, causal=False, out_dtype=dtype)
        per = rows.shape[1] // 8
        for h in range(0, rows.shape[1], 3):
            one = rows[0, h].float().numpy()
            y64, off = row64(one, k[:, h // per], v[:, h // per], hblock, dim ** -0.5, fine)
            (ck, sk), (cv, sv) = ([x.astype(np.float64) for x in quantize(x[:, h // per], hblock)] for x in (k, v))
            t = (ck * sk) @ butterfly(one.astype(np.float64), hblock) * (dim ** -0.5 / hblock)
            w = np.exp(t - t.max()) / np.exp(t - t.max()).sum()
            qt = np.abs(butterfly(one.astype(np.float64), hblock)).max()
            more = np.expm1(2 * 2.0 ** -38 * qt * np.abs(ck * sk).sum(1).max() * (dim ** -0.5 / hblock))
            off = off + more * butterfly_abs((w @ np.abs(cv * sv))[None], hblock)[0]
            check(y[0, h].cpu(), y64, off, f"head {h} of {rows.shape[1]}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_that_grow(dtype):
    """Every step's largest weight a little or a lot above the one before."""
    for nats in (0.5, 2.0, 5.0, 9.0):
        s = Sequences([640], 8, 128, 64, 64, torch.float32, seed=int(10 * nats), poison=False)
        s.k *= 0.05
        s.k[:, :, 0] = torch.arange(640)[:, None] // 32 * nats / 4.0        # (the transform spreads it over its 64 channels)
        q = torch.zeros((1, 16, 128), dtype=dtype)
        q[..., 0] = 4.0 * 128 ** 0.5
        run(s, q, dtype != torch.bfloat16, dtype, 1)
