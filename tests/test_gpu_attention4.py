"""Attention over the 4-bit cache against a plain implementation in 64 bits on the values
that the cache holds; the tolerance is derived at cache4_util.attention64.

Head sizes, grouped heads, pages, lengths from none to many, one new token, a few and
parts of prompts, ragged rows, windows, absent pages, types and strides, values far from
one, and what may lie in positions that are not seen."""
import numpy as np
import pytest
import torch

from cache4_util import Sequences, attention64, check, held, most_scale
from gpu_util import DEV, Guarded, dev, host
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def queries(s, new, q_heads, dtype, size=1.0):
    q = s.rng.normal(size=(sum(new), q_heads, s.dim)) * size
    return torch.from_numpy(q.astype(np.float32)).to(dtype)


def compare(s, q, new, y, causal=True, window=0, scale=None, what="", there=None):
    scale = s.dim ** -0.5 if scale is None else scale
    fine = not (q.dtype == torch.bfloat16 and y.dtype == torch.bfloat16)
    row = 0
    for i, n in enumerate(new):
        k, v = s.of(i)
        y64, bound = attention64(q[row:row + n].float().numpy(), held(k, s.hblock), held(v, s.hblock), most_scale(v, s.hblock), s.hblock, np.float32(scale).astype(np.float64), causal,
                                 window, fine, None if there is None else there[i])
        check(y[row:row + n].cpu(), y64, bound, f"{what} sequence {i} of {len(new)}, length {s.lens_np[i]}, {n} rows")
        row += n


def run(s, new, share, dtype, causal=True, window=0, size=1.0, even=False, **kw):
    q = queries(s, new, s.heads * share, dtype, size)
    ends = None if even else dev(np.cumsum(new).astype(np.int32))
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, ends=ends, causal=causal, window=window, **kw)
    assert y.shape == q.shape
    compare(s, q, new, y, causal, window, kw.get("scale"))
    return q, y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,hblock,heads,share,page", [(128, 128, 2, 4, 64), (64, 64, 3, 1, 16), (80, 16, 1, 5, 32), (32, 32, 2, 8, 16),
                                                         (256, 64, 1, 2, 16), (192, 64, 2, 3, 64), (1, 1, 1, 1, 16), (97, 1, 1, 16, 16),
                                                         (128, 1, 1, 17, 256), (72, 8, 2, 33, 16), (224, 32, 1, 4, 64), (256, 128, 1, 1, 16)])
def test_one_token(dim, hblock, heads, share, page, dtype):
    """A step of a batch: lengths around the tiles' and pages' ends."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 257, 300]
    s = Sequences(lens, heads, dim, hblock, page, dtype, seed=dim + share)
    s.write()
    run(s, [1] * len(lens), share, dtype, even=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[1000], [2049, 5], [513, 700, 1, 32]])
def test_long(lens, dtype):
    s = Sequences(lens, 2, 128, 128, 64, dtype, seed=len(lens))
    s.write()
    run(s, [1] * len(lens), 4, dtype, even=True, size=3.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 20), (True, 33), (True, 2 ** 31 - 1)])
@pytest.mark.parametrize("new", [[3, 1, 5, 2], [17, 40, 0, 33], [0, 0, 7, 0]])
def test_a_few_tokens(new, causal, window, dtype):
    s = Sequences([90, 41, 7, 200], 2, 64, 64, 16, dtype, seed=sum(new))
    s.write()
    run(s, new, 3, dtype, causal, window)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,hblock,share", [(128, 128, 8), (64, 64, 5), (80, 16, 4), (192, 64, 8), (256, 128, 8)])
def test_parts_of_prompts(dim, hblock, share, dtype):
    """Rows enough for the kernel that gives each wave columns of its own."""
    new = [130, 7, 0, 201]
    s = Sequences([130, 60, 33, 290], 2, dim, hblock, 32, dtype, seed=dim)
    s.write()
    for causal, window in ((True, 0), (True, 70), (False, 0)):
        run(s, new, share, dtype, causal, window)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim,hblock", [(64, 64), (40, 8), (128, 128), (80, 16), (192, 64), (136, 8)])
def test_blocks_of_many_columns(dim, hblock, page, dtype):
    """Rows enough for blocks of 32, 48 or 64 columns, of which there have to be 512."""
    new = [130, 7, 0, 370, 1]
    s = Sequences([130, 60, 33, 400, 65], 8, dim, hblock, page, dtype, seed=dim + page)
    s.write()
    for causal, window in ((True, 0), (True, 70), (False, 0)):
        run(s, new, 8, dtype, causal, window)


def test_blocks_of_many_columns_absent_pages_and_nan():
    new = [400, 100]
    s = Sequences([450, 100], 8, 128, 64, 16, torch.bfloat16, seed=5)
    s.k[50, 3], s.v[450 + 20, 5, 1] = float("nan"), float("inf")
    s.write()
    table, there = s.table_np.copy(), [np.ones(450, bool), np.ones(100, bool)]
    for i, p in ((0, 1), (0, 17), (1, 0), (1, 6)):
        table[i, p] = [-1, s.cache.pages][p & 1]
        there[i][16 * p:16 * p + 16] = False
    q = queries(s, new, 64, torch.bfloat16)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), dev(table), s.lens, ends=dev(np.cumsum(new).astype(np.int32)))
    compare(s, q, new, y, there=there)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_even_prompts(dtype):
    s = Sequences([96, 96, 96], 1, 64, 64, 16, dtype, seed=4)
    s.write()
    run(s, [96] * 3, 4, dtype, even=True)
    run(s, [96] * 3, 1, dtype, even=True)


@pytest.mark.parametrize("rows", ["one", "many"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_see_nothing(rows, dtype):
    """Lengths of none, and more rows than positions: 0, not NaN."""
    s = Sequences([0, 3, 50, 0], 1, 64, 64, 16, dtype, seed=8)
    s.write()
    new = [1, 5, 1, 2] if rows == "one" else [90, 300, 70, 100]
    q, y = run(s, new, 4, dtype)
    assert bool((y[:new[0]] == 0).all()) and bool((y[new[0]:new[0] + new[1] - 3] == 0).all())
    s = Sequences([0], 1, 64, 64, 16, dtype, seed=8)
    y = hatq.hatq_attention4(s.cache, queries(s, [3], 2, dtype).to(DEV), s.table, s.lens, causal=False)
    assert bool((y == 0).all())


@pytest.mark.parametrize("new", [1, 100])
def test_absent_pages(new):
    """Positions of pages that the cache does not have are not seen."""
    s = Sequences([150, 150], 2, 64, 64, 16, torch.float32, seed=21)
    s.write()
    table = s.table_np.copy()
    table[0, [0, 3, 4, 9]] = [-1, 2 ** 31 - 1, -2 ** 31, s.cache.pages]
    table[1, :] = -7
    there = [np.ones(150, bool), np.zeros(150, bool)]
    for p in (0, 3, 4, 9):
        there[0][16 * p:16 * p + 16] = False
    q = queries(s, [new] * 2, 8, torch.float32)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), dev(table), s.lens)
    compare(s, q, [new] * 2, y, there=there)
    assert bool((y[new:] == 0).all())
    # a length past the table's width ends there
    y = hatq.hatq_attention4(s.cache, q[:new].to(DEV), s.table[:1, :4].contiguous(), dev(np.array([2 ** 31 - 1], np.int32)), causal=False)
    there = np.arange(150) < 64
    compare(s, q[:new], [new], y, causal=False, there=[there])


@pytest.mark.parametrize("new,window", [(1, 0), (6, 0), (100, 0), (100, 20), (6, 30), (150, 7)])
@pytest.mark.parametrize("page,share", [(16, 4), (32, 1), (16, 1)])
def test_lengths_past_the_table(new, window, page, share):
    """A row's position counts from its sequence's length, also where that is past the table:
    it sees the table's positions before its own."""
    s = Sequences([150], 2, 128, 64, page, torch.float32, seed=22)
    s.write()
    width = 80 // page
    q = queries(s, [new], 2 * share, torch.float32)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table[:, :width].contiguous(), s.lens, window=window)
    there = np.arange(150) < width * page
    compare(s, q, [new], y, window=window, there=[there])


def test_the_longest_length():
    s = Sequences([64], 1, 64, 64, 16, torch.bfloat16, seed=23)
    s.write()
    q = queries(s, [2], 1, torch.bfloat16).to(DEV)
    long = dev(np.array([2 ** 31 - 1], np.int32))
    y = hatq.hatq_attention4(s.cache, q, s.table, long)
    assert torch.equal(y, hatq.hatq_attention4(s.cache, q, s.table, s.lens, causal=False))
    assert bool((hatq.hatq_attention4(s.cache, q, s.table, long, window=2 ** 31 - 1 - 2 ** 30) == 0).all())
    assert bool((hatq.hatq_attention4(s.cache, q, s.table, long, window=1) == 0).all())
    assert torch.equal(y, hatq.hatq_attention4(s.cache, q, s.table, long, window=2 ** 31 - 1))
    none = dev(np.array([0], np.int32))
    assert bool((hatq.hatq_attention4(s.cache, q, s.table, none, window=2 ** 31 - 1) == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite(dtype):
    """A NaN key or value in one sequence makes its own rows NaN that see it, no others; what
    lies in hidden positions does nothing."""
    s = Sequences([40, 40, 40], 1, 64, 64, 16, dtype, seed=31)
    s.k[5], s.v[40 + 20, 0, 3] = float("nan"), float("inf")
    s.write()
    q = queries(s, [40] * 3, 8, dtype)
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)
    nan = torch.isnan(y).all(-1).all(-1).cpu().numpy()
    some = torch.isnan(y).any(-1).any(-1).cpu().numpy()
    want = np.zeros(120, bool)
    want[5:40] = want[60:80] = True
    assert (nan == want).all() and (some == want).all()
    # a query that is not finite: its row alone, and its head
    q[85, 2, 7] = float("inf")
    y = torch.isnan(hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)).all(-1)
    assert bool(y[85, 2]) and int(y[80:].sum()) == 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k_scale,v_scale,size", [(1e-3, 1e20, 1e3), (1.0, 1e-20, 1.0), (1e15, 1.0, 1e-15), (1.0, 1e-30, 30.0), (1.0, 1e30, 30.0),
                                                  (1e-20, 1.0, 1.0)])
def test_far_from_one(k_scale, v_scale, size, dtype):
    s = Sequences([70, 33], 2, 64, 64, 16, dtype, seed=41, k_scale=k_scale, v_scale=v_scale)
    # values of one sequence spread over 10 orders of magnitude, a zero one among them
    s.v[:70] *= torch.from_numpy((10.0 ** np.linspace(-5, 5, 70)).astype(np.float32))[:, None, None].to(dtype)
    s.v[12] = 0
    s.write()
    run(s, [1, 1], 2, dtype, size=size)
    run(s, [70, 33], 8, dtype, size=size)


def test_a_small_value_with_all_the_weight():
    """The first position has nearly all the weight and a tiny value; the others' values are
    large: both count."""
    s = Sequences([65], 1, 64, 64, 16, torch.float32, seed=51)
    s.k[0] = s.k[0].abs() * 8
    s.v[0] *= 1e-6
    s.v[1:] *= 1e4
    s.write()
    q = torch.ones((1, 1, 64)) * 0.5
    y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)
    compare(s, q, [1], y)


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float16, torch.float16)])
def test_strides_and_types(dtype, out):
    s = Sequences([33, 80], 2, 72, 8, 16, torch.bfloat16, seed=61)
    s.write()
    q = queries(s, [2, 2], 6, dtype)
    wide = torch.zeros((4, 7 * 72 + 3), dtype=dtype, device=DEV)
    view = wide[:, 3:3 + 6 * 72].unflatten(1, (6, 72))
    view.copy_(q)
    y_wide = torch.full((6, 4, 72 + 5), 9.0, dtype=out, device=DEV)
    y = y_wide[:, :, 5:].transpose(0, 1)
    got = hatq.hatq_attention4(s.cache, view, s.table, s.lens, scale=0.2, y=y)
    assert got is y
    compare(s, q, [2, 2], y, scale=0.2)
    assert bool((y_wide[:, :, :5] == 9).all())
    # one query for all rows
    one = q[:1].to(DEV).expand(4, 6, 72)
    y = hatq.hatq_attention4(s.cache, one, s.table, s.lens, out_dtype=out)
    compare(s, one.cpu(), [2, 2], y)


def test_rows_past_the_last_end():
    s = Sequences([33, 80], 1, 64, 64, 16, torch.float32, seed=71)
    s.write()
    for new, rows in (([1, 2], 5), ([33, 80], 140)):
        q = queries(s, [rows], 8, torch.float32)
        ends = dev(np.cumsum(new).astype(np.int32))
        g = Guarded((rows, 8, 64), torch.float32)
        g.view.fill_(3.0)
        hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, ends=ends, y=g.view)
        g.check()
        assert bool((g.view[sum(new):] == 3).all())
        compare(s, q[:sum(new)], new, g.view[:sum(new)].clone())


def test_any_ends_lens_and_tables_are_safe():
    rng = np.random.default_rng(2)
    s = Sequences([60, 60, 60, 60, 60], 1, 64, 64, 16, torch.float32, seed=72)
    s.write()
    for rows in (30, 400):
        q = torch.ones((rows, 4, 64), device=DEV)
        for _ in range(15):
            big = rng.integers(-2 ** 31, 2 ** 31, size=(2, 5)).astype(np.int32)
            small = rng.integers(-3, rows + 30, size=(2, 5)).astype(np.int32)
            pick = np.where(rng.random((2, 5)) < 0.5, big, small)
            table = dev(np.where(rng.random((5, 4)) < 0.3, rng.integers(-2 ** 31, 2 ** 31, size=(5, 4)), s.table_np[:, :4]).astype(np.int32))
            g = Guarded((rows, 4, 64), torch.float32)
            hatq.hatq_attention4(s.cache, q, table, dev(pick[0]), ends=dev(pick[1]), y=g.view, window=int(rng.integers(0, 50)))
            g.check()


@pytest.mark.parametrize("dtype,lens", [(torch.bfloat16, 3000), (torch.float32, 3000), (torch.bfloat16, 9000), (torch.float32, 9000)])
def test_splits(dtype, lens):
    """One sequence over many blocks: every choice of the launch gives the sums, the same
    bits each time; the workspace is as large as asked for and not larger."""
    s = Sequences([lens, 17], 1, 128, 64, 16, dtype, seed=81)
    s.write()
    q = queries(s, [1, 1], 4, dtype)
    sizes = set()
    for max_len in (0, 1, 600, 1500, 3000, 5000, 2 ** 31 - 1):
        n = hatq.hatq_attention4_ws_bytes(s.cache, 2, 4, s.table.shape[1], 2, False, 0, max_len)
        sizes.add(n)
        g = Guarded((max(n, 256),), torch.int8)
        y = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, max_len=max_len, ws=g.view)
        g.check("workspace")
        compare(s, q, [1, 1], y)
        again = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, max_len=max_len)
        assert torch.equal(y, again)
        if n:
            with pytest.raises(hatq.HatqError) as e:
                hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens, max_len=max_len, ws=g.view[:n - 256])
            assert e.value.status == hatq.HATQ_EWORKSPACE
    assert 0 in sizes and len(sizes) > (1 if lens == 3000 else 3)


def test_past_32_bits():
    heads, dim, page = 16, 128, 256
    pages = 2 ** 32 // (heads * page * 2 * 68) + 40
    cache = hatq.hatq_cache4_init(pages, page, heads, dim, hblock=128, device=DEV)
    assert cache.buf.numel() > 2 ** 32
    s = Sequences([page + 40], heads, dim, 128, page, torch.bfloat16, seed=91, spare=0)
    s.cache, s.table = cache, dev(np.array([[pages - 1, pages - 3]], np.int32))
    s.write()
    run(s, [1], 2, torch.bfloat16)
    run(s, [100], 4, torch.bfloat16)
    del cache, s
    torch.cuda.empty_cache()


def test_a_step_captured_and_replayed():
    """Append and attention as one graph, replayed with new tokens and lengths between
    eager calls; other streams' workspaces are their own."""
    dtype = torch.bfloat16
    s = Sequences([700, 300], 2, 128, 128, 64, dtype, seed=95)
    s.write()
    lens = dev(np.array([600, 200], np.int32))
    k, v = (torch.zeros((2, 2, 128), dtype=dtype, device=DEV) for _ in range(2))
    q = torch.zeros((2, 8, 128), dtype=dtype, device=DEV)
    y = torch.zeros_like(q)
    ws = torch.empty(max(256, hatq.hatq_attention4_ws_bytes(s.cache, 2, 8, s.table.shape[1], 2)), dtype=torch.int8, device=DEV)

    def step(out):
        hatq.hatq_cache4_append(s.cache, k, v, s.table, lens)
        hatq.hatq_attention4(s.cache, q, s.table, lens, y=out, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y)
    for i in range(4):
        lens += 1
        k.copy_(torch.randn((2, 2, 128)))
        v.copy_(torch.randn((2, 2, 128)))
        q.copy_(torch.randn((2, 8, 128)))
        graph.replay()
        other = torch.zeros_like(y)
        eager = hatq.hatq_attention4(s.cache, q, s.table, lens, y=other)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        got = hatq.hatq_cache4_read(s.cache, 2, s.table, lens)[0]
        want = torch.from_numpy(held(k.float().cpu().numpy(), 128)).to(DEV)
        step_ = torch.from_numpy(np.abs(want.cpu().numpy()).max(-1, keepdims=True)).to(DEV)
        assert bool(((got - k.float()).abs() <= step_).all())


def test_another_stream():
    s = Sequences([700], 2, 64, 64, 16, torch.float32, seed=96)
    s.write()
    q = queries(s, [1], 4, torch.float32).to(DEV)
    here = hatq.hatq_attention4(s.cache, q, s.table, s.lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = hatq.hatq_attention4(s.cache, q, s.table, s.lens, stream=side)
    side.synchronize()
    assert torch.equal(here, there)


def test_pages_that_sequences_share():
    """Sequences with the same first pages read them as if each had its own."""
    s = Sequences([96, 80], 2, 64, 64, 16, torch.bfloat16, seed=101)
    s.k[96:160], s.v[96:160] = s.k[:64].clone(), s.v[:64].clone()
    s.write()
    q = queries(s, [5, 5], 4, torch.bfloat16)
    own = hatq.hatq_attention4(s.cache, q.to(DEV), s.table, s.lens)
    table = s.table_np.copy()
    table[1, :4] = table[0, :4]
    assert torch.equal(own, hatq.hatq_attention4(s.cache, q.to(DEV), dev(table), s.lens))
    table[0, 4] = table[0, 5]       # the same page twice in one sequence: its positions twice
    y = hatq.hatq_attention4(s.cache, q.to(DEV), dev(table), s.lens, causal=False)
    at = 5 * 16
    s.k[64:80], s.v[64:80] = s.k[at:at + 16].clone(), s.v[at:at + 16].clone()
    compare(s, q, [5, 5], y, causal=False)


@pytest.mark.parametrize("lens,new", [([3000, 2900], 1), ([300, 200], 40), ([5000], 3)])
def test_into_the_queries(lens, new):
    """Results may take the queries' place."""
    s = Sequences(lens, 2, 128, 64, 64, torch.bfloat16, seed=102)
    s.write()
    q = queries(s, [new] * len(lens), 8, torch.bfloat16).to(DEV)
    y = hatq.hatq_attention4(s.cache, q, s.table, s.lens)
    assert hatq.hatq_attention4(s.cache, q, s.table, s.lens, y=q) is q
    assert torch.equal(q, y)


def test_two_calls_at_once():
    """Two streams, each with its own workspace (which a call makes itself)."""
    s = Sequences([20000, 9000], 2, 128, 64, 64, torch.float16, seed=103)
    s.write()
    q = [queries(s, [1, 1], 16, torch.float16).to(DEV) for _ in range(2)]
    alone = [hatq.hatq_attention4(s.cache, x, s.table, s.lens) for x in q]
    assert hatq.hatq_attention4_ws_bytes(s.cache, 2, 16, s.table.shape[1], 2) > 0
    side = [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    for _ in range(5):
        both = [hatq.hatq_attention4(s.cache, x, s.table, s.lens, stream=st) for x, st in zip(q, side)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(alone, both))


def test_refusals():
    s = Sequences([30, 30], 2, 64, 64, 16, torch.float32, seed=97)
    s.write()
    q = torch.zeros((2, 4, 64), device=DEV)
    ok = dict(causal=True)
    hatq.hatq_attention4(s.cache, q, s.table, s.lens, **ok)

    def bad(*a, **k):
        with pytest.raises((ValueError, hatq.HatqError)):
            hatq.hatq_attention4(*a, **k)
    bad(s.cache, q[:, :3], s.table, s.lens)                 # 3 query heads over 2
    bad(s.cache, q[:, :, :32], s.table, s.lens)
    bad(s.cache, q[:1], s.table, s.lens)                    # 1 row of 2 sequences
    bad(s.cache, q, s.table.long(), s.lens)
    bad(s.cache, q, s.table, s.lens[:1])
    bad(s.cache, q, s.table, s.lens, window=-1)
    bad(s.cache, q, s.table, s.lens, window=4, causal=False)
    bad(s.cache, q, s.table, s.lens, scale=float("nan"))
    bad(s.cache, q, s.table, s.lens, max_len=-1)
    bad(s.cache, q, s.table, s.lens, max_len=2 ** 31)
    bad(s.cache, q, s.table, s.lens, y=torch.zeros((2, 4, 63), device=DEV))
    bad(s.cache, q, s.table, s.lens, y=torch.zeros((1, 4, 64), device=DEV).expand(2, 4, 64))
    bad(s.cache, q, s.table, s.lens, out_dtype=torch.float64)
    bad(s.cache, q.cpu(), s.table, s.lens)
    bad(s.cache, q, s.table.cpu(), s.lens)
    assert hatq.hatq_attention4(s.cache, q[:0], s.table, s.lens).shape == (0, 4, 64)
