"""Attention over the 4-bit cache where a sequence's positions are dealt to several blocks and
joined: every number of 64-channel blocks of a head and both kinds of pages, ragged rows,
windows, masks, pages and keys that are missing or not finite, and parts that hold no position.
The tolerance is cache4_util.attention64's."""
import numpy as np
import pytest
import torch

from cache4_util import Sequences
from gpu_util import DEV, Guarded, dev
from paper_2608_01653_amd import hatq
from test_gpu_attention4 import compare, queries

pytestmark = pytest.mark.gpu
HEADS = [(64, 64), (80, 16), (128, 128), (192, 64), (256, 128), (40, 8)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def parts(s, rows, q_heads, **kw):
    """Whether the call's positions are dealt to several blocks."""
    return hatq.hatq_attention4_ws_bytes(s.cache, rows, q_heads, s.table.shape[1], len(s.lens_np), **kw) > 0


def same(a, b):
    """Equal, NaN among the values."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))


def ragged(s, new, share, dtype, past=0, table=None, there=None, **kw):
    """Rows of unlike sequences, `past` more behind the last end, which stay as they are."""
    rows, q_heads = sum(new), s.heads * share
    q = queries(s, new, q_heads, dtype)
    assert parts(s, rows + past, q_heads, ragged=True, window=kw.get("window", 0))
    y = Guarded((rows + past, q_heads, s.dim), dtype)
    y.view.fill_(9.0)
    wide = torch.cat((q, torch.ones((past, q_heads, s.dim), dtype=dtype))).to(DEV)
    ends = dev(np.cumsum(new).astype(np.int32))
    table = s.table if table is None else table
    hatq.hatq_attention4(s.cache, wide, table, s.lens, ends=ends, y=y.view, **kw)
    y.check()
    assert bool((y.view[rows:] == 9).all())
    got = y.view[:rows].clone()
    compare(s, q, new, got, kw.get("causal", True), kw.get("window", 0), there=there)
    # the same bits again, and into the queries' place
    assert same(got, hatq.hatq_attention4(s.cache, wide, table, s.lens, ends=ends, **kw)[:rows])
    hatq.hatq_attention4(s.cache, wide, table, s.lens, ends=ends, y=wide, **kw)
    assert same(got, wide[:rows]) and bool((wide[rows:] == 1).all())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim,hblock", HEADS)
@pytest.mark.parametrize("kw", [dict(), dict(window=1100), dict(causal=False)])
def test_ragged_rows(kw, dim, hblock, page, dtype):
    """An empty sequence, one far shorter than the longest (most of its parts are empty), and
    rows behind the last end."""
    s = Sequences([3000, 0, 1500, 20], 2, dim, hblock, page, dtype, seed=dim + page)
    s.write()
    ragged(s, [2, 1, 3, 1], 2, dtype, past=2, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim,hblock", HEADS)
def test_absent_pages_and_not_finite(dim, hblock, page, dtype):
    """Whole parts of absent pages, single ones at a part's ends, a key and a value of one part
    that are not finite."""
    lens = [2050, 1800, 1300]
    s = Sequences(lens, 1, dim, hblock, page, dtype, seed=dim)
    s.k[2050 + 900, 0, 3], s.v[2050 + 1800 + 1299, 0, dim - 1] = float("nan"), float("inf")
    s.write()
    table, there = s.table_np.copy(), [np.ones(n, bool) for n in lens]
    for i, (first, last) in ((0, (0, 640)), (0, (1024, 1088)), (0, (1984, 2050)), (2, (512, 1024))):
        for p in range(first // page, -(-last // page)):
            table[i, p] = [-1, s.cache.pages, 2 ** 31 - 1][p % 3]
            there[i][page * p:page * (p + 1)] = False
    got = ragged(s, [2, 3, 2], 3, dtype, table=dev(table), there=there)
    # the NaN key's sequence: all three rows; the value's: only the last position's row sees it
    assert bool(torch.isnan(got[2:5]).all()) and bool(torch.isnan(got[6]).all()) and not bool(torch.isnan(got[[0, 1, 5]]).any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("dim,hblock", [(64, 64), (72, 8), (128, 128), (192, 64)])
def test_many_steps_a_block(dim, hblock, page, dtype):
    """Two parts of each sequence, of 64 steps and more: 16 waves a block up to 128 channels."""
    lens = [4100, 3, 33, 0, 1, 2048, 16, 17] + [5] * 8
    s = Sequences(lens, 8, dim, hblock, page, dtype, seed=dim + page)
    s.write()
    q = queries(s, [1] * 16, 16, dtype)
    assert parts(s, 16, 16)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)
    compare(s, q, [1] * 16, y)
    assert bool((y[3] == 0).all())


@pytest.mark.parametrize("page,dim", [(16, 64), (64, 256), (16, 256)])
def test_columns_of_several_tiles(page, dim):
    """More columns of a head than one block takes, and sequences of fewer positions than rows."""
    s = Sequences([1100, 4], 1, dim, 64, page, torch.float32, seed=page)
    s.write()
    got = ragged(s, [7, 6], 5, torch.float32, past=1)
    assert bool((got[7:9] == 0).all()) and not bool((got[9:] == 0).all())


def test_captured_and_replayed():
    """Parts joined in a graph, the workspace its own, lengths and rows changed between replays."""
    s = Sequences([2600, 1900], 1, 80, 16, 16, torch.float32, seed=7)
    s.write()
    q = queries(s, [2, 2], 3, torch.float32).to(DEV)
    lens, ends = s.lens.clone(), dev(np.array([2, 4], np.int32))
    n = hatq.hatq_attention4_ws_bytes(s.cache, 4, 3, s.table.shape[1], 2, True)
    assert n > 0
    ws, y = torch.empty(n, dtype=torch.int8, device=DEV), torch.zeros_like(q)
    hatq.hatq_attention4(s.cache, q, s.table, lens, ends=ends, y=y, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hatq.hatq_attention4(s.cache, q, s.table, lens, ends=ends, y=y, ws=ws)
    for i, (a, b, end) in enumerate([(2600, 1900, 2), (40, 1900, 1), (2600, 0, 3), (1, 2, 2), (2599, 1024, 4)]):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        ends[0] = end
        ws.fill_(i)
        graph.replay()
        eager = hatq.hatq_attention4(s.cache, q, s.table, lens, ends=ends, y=torch.zeros_like(q))
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
