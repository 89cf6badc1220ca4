"""The 4-bit cache of keys and values: what is written and read back, bit for bit against
the same arithmetic in numpy (float32 sums, products and divisions in a fixed order and
the rounding of a scale to bfloat16 are the same everywhere), over head sizes, transform
blocks, pages, types, strides and ragged rows, and what is left out."""
import numpy as np
import pytest
import torch

from cache4_util import Sequences, butterfly, held, quantize
from gpu_util import DEV, Guarded, dev, host
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def read_back(x, hblock):
    """Heads as the cache gives them back, float32: float32 products and sums."""
    q, s = quantize(x, hblock)
    with np.errstate(all="ignore"):
        return butterfly(q.astype(np.float32) * s, hblock) * np.float32(1.0 / hblock)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("dim,hblock", [(128, 128), (128, 64), (64, 64), (64, 1), (80, 16), (1, 1), (7, 1), (96, 32), (33, 1),
                                        (192, 64), (256, 128), (256, 8), (200, 8), (48, 2), (36, 4)])
def test_round_trip(dim, hblock, dtype):
    s = Sequences([37, 1, 0, 16, 130], 3, dim, hblock, 16, dtype, seed=dim * hblock)
    s.write()
    ends = dev(np.cumsum(s.lens_np).astype(np.int32))
    for out in (torch.float32, dtype):
        k, v = hatq.hatq_cache4_read(s.cache, sum(s.lens_np), s.table, s.lens, ends=ends, out_dtype=out)
        for got, x in ((k, s.k), (v, s.v)):
            want = torch.from_numpy(read_back(x.float().numpy(), hblock)).to(out)
            assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("page", [16, 32, 256, 65536])
def test_pages_and_steps(page):
    """A sequence written in parts, one token at a time among them, is the one written at once."""
    one, parts = (Sequences([75, 300], 2, 64, 64, page, torch.bfloat16, seed=5, spare=2) for _ in range(2))
    one.write()
    first = [40, 299]
    rows = [np.arange(0, 40), 75 + np.arange(299)]
    ends = dev(np.cumsum(first).astype(np.int32))
    pick = np.concatenate(rows)
    hatq.hatq_cache4_append(parts.cache, parts.k[pick].to(DEV), parts.v[pick].to(DEV), parts.table, dev(np.array(first, np.int32)), ends=ends)
    # one token each, then the rest of the first alone
    step = np.array([40, 75 + 299])
    hatq.hatq_cache4_append(parts.cache, parts.k[step].to(DEV), parts.v[step].to(DEV), parts.table, dev(np.array([41, 300], np.int32)))
    rest = np.arange(41, 75)
    hatq.hatq_cache4_append(parts.cache, parts.k[rest].to(DEV), parts.v[rest].to(DEV), parts.table[:1], parts.lens[:1])
    assert torch.equal(one.cache.buf, parts.cache.buf)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dtype):
    """Keys and values inside the rows of a wider product, heads before rows, odd offsets."""
    rng = np.random.default_rng(3)
    lens = dev(np.array([20, 20], np.int32))
    table = dev(np.array([[1, 3], [0, 2]], np.int32))
    wide = torch.from_numpy(rng.normal(size=(40, 9 * 72 + 1)).astype(np.float32)).to(dtype).to(DEV)
    k = wide[:, 1:1 + 3 * 72].unflatten(1, (3, 72))
    v = wide[:, 1 + 6 * 72:].unflatten(1, (3, 72)).transpose(0, 1).contiguous().transpose(0, 1)
    assert v.stride(0) == 72
    cache = hatq.hatq_cache4_init(4, 16, 3, 72, hblock=8, device=DEV)
    hatq.hatq_cache4_append(cache, k, v, table, lens)
    wide_out = torch.full((40, 3 * 72 + 5), 7.0, dtype=dtype, device=DEV)
    k_out = wide_out[:, 3:3 + 3 * 72].unflatten(1, (3, 72))
    v_out = torch.empty((3, 40, 72), dtype=dtype, device=DEV).transpose(0, 1)
    hatq.hatq_cache4_read(cache, 40, table, lens, k=k_out, v=v_out)
    for got, x in ((k_out, k), (v_out, v)):
        assert torch.equal(got.cpu(), torch.from_numpy(read_back(x.float().cpu().numpy(), 8)).to(dtype))
    assert bool((wide_out[:, :3] == 7).all()) and bool((wide_out[:, 3 + 3 * 72:] == 7).all())


def test_values_at_the_ends_of_the_range():
    """Zeros, subnormals, the largest, ties between codes, infinities and NaN."""
    x = np.zeros((16, 1, 64), np.float32)
    x[1] = 1e-45
    x[2, 0, :] = np.linspace(-3e38, 3e38, 64)
    x[3, 0, ::2], x[3, 0, 1::2] = 7.0, np.arange(32) % 15 - 7.5      # s = 1: halves
    x[4, 0, 5] = np.inf
    x[5, 0, 60] = np.nan
    x[6, 0, 0] = -np.inf
    x[7] = 1.17e-38
    x[8, 0, :] = np.linspace(-1e-40, 1e-40, 64)
    x[9, 0, 3] = 1.0
    x[10, 0, :8] = [2.0 ** -k for k in range(8)]
    x[11] = -0.0
    x[12] = 1e30
    x[13, 0, 0], x[13, 0, 1] = 2.0 ** 102, 5.0
    x[14, 0, 0], x[14, 0, 1] = np.nextafter(np.float32(2.0 ** 102), np.float32(0)), 2.0 ** 99
    x[15, 0, :] = np.linspace(-3e-30, 3e-30, 64)
    for hblock in (1, 64):
        cache = hatq.hatq_cache4_init(1, 16, 1, 64, hblock=hblock, device=DEV)
        place = dev(np.zeros((1, 1), np.int32)), dev(np.array([16], np.int32))
        hatq.hatq_cache4_append(cache, dev(x), dev(x), *place)
        k, v = hatq.hatq_cache4_read(cache, 16, *place)
        want = read_back(x, hblock)
        for got in (host(k), host(v)):
            np.testing.assert_array_equal(got, want)


def test_what_is_left_out():
    """Absent pages, positions before the first and past the table, rows past the last end."""
    rng = np.random.default_rng(9)
    heads, dim = 2, 64
    x = rng.normal(size=(60, heads, dim)).astype(np.float32)
    cache = hatq.hatq_cache4_init(3, 16, heads, dim, hblock=64, device=DEV)
    guard = Guarded((cache.buf.numel(),), torch.int8)
    guard.view.fill_(0x11)
    cache = hatq.hatq_cache4_init(3, 16, heads, dim, hblock=64, buf=guard.view)
    # 32 positions, the second page absent; past the table's 32; 4 rows of which 2 before 0
    table = dev(np.array([[2, -1], [0, 3], [1, 2 ** 31 - 1]], np.int32))
    lens = dev(np.array([32, 40, 2], np.int32))
    ends = dev(np.array([32, 52, 56], np.int32))
    hatq.hatq_cache4_append(cache, dev(x), dev(x), table, lens, ends=ends)
    k = torch.full((60, heads, dim), 5.0, device=DEV)
    v = k.clone()
    hatq.hatq_cache4_read(cache, 60, table, lens, ends=ends, k=k, v=v)
    guard.check("cache")
    want = read_back(x, 64)
    want[16:32] = 0            # absent
    want[32:52] = 0            # positions 20 .. 39: page 3 of 3, then past the table
    want[52:54] = 0            # positions -2, -1
    want[56:] = 5.0            # past the last end
    for got in (host(k), host(v)):
        np.testing.assert_array_equal(got, want)
    # pages 0 and the rest of page 1 have not been written
    per = cache.buf.numel() // 3
    assert bool((cache.buf[:per] == 0x11).all())


def test_any_ends_lens_and_tables_are_safe():
    rng = np.random.default_rng(2)
    cache0 = hatq.hatq_cache4_init(4, 16, 1, 64, device=DEV)
    guard = Guarded((cache0.buf.numel(),), torch.int8)
    cache = hatq.hatq_cache4_init(4, 16, 1, 64, buf=guard.view)
    x = torch.ones((30, 1, 64), device=DEV)
    for _ in range(20):
        big = rng.integers(-2 ** 31, 2 ** 31, size=(3, 5)).astype(np.int32)
        small = rng.integers(-3, 40, size=(3, 5)).astype(np.int32)
        pick = np.where(rng.random((3, 5)) < 0.5, big, small)
        out = Guarded((30, 1, 64), torch.float32)
        table = dev(np.where(rng.random((5, 2)) < 0.3, 2 ** 30, rng.integers(-1, 5, size=(5, 2))).astype(np.int32))
        hatq.hatq_cache4_append(cache, x, x, table, dev(pick[0]), ends=dev(pick[1]))
        hatq.hatq_cache4_read(cache, 30, table, dev(pick[0]), ends=dev(pick[1]), k=out.view, v=torch.empty_like(x))
        out.check()
        guard.check()


def test_past_32_bits():
    """Pages that lie more than 2^32 bytes into the cache."""
    heads, dim, page = 16, 256, 256
    pages = 2 ** 32 // (heads * page * 4 * 68) + 40
    cache = hatq.hatq_cache4_init(pages, page, heads, dim, hblock=128, device=DEV)
    assert cache.buf.numel() > 2 ** 32
    x = torch.randn((page + 3, heads, dim), device=DEV)
    table, lens = dev(np.array([[pages - 1, pages - 2]], np.int32)), dev(np.array([page + 3], np.int32))
    hatq.hatq_cache4_append(cache, x, -x, table, lens)
    k, v = hatq.hatq_cache4_read(cache, page + 3, table, lens)
    want = read_back(host(x), 128)
    np.testing.assert_array_equal(host(k), want)
    np.testing.assert_array_equal(host(v), -want)
    del cache, x, k, v
    torch.cuda.empty_cache()


def test_refusals():
    cache = hatq.hatq_cache4_init(4, 16, 2, 64, device=DEV)
    x = torch.zeros((4, 2, 64), device=DEV)
    table, lens = dev(np.zeros((2, 1), np.int32)), dev(np.array([2, 2], np.int32))
    def bad(*a, **k):
        with pytest.raises((ValueError, hatq.HatqError)):
            hatq.hatq_cache4_append(*a, **k)
    bad(cache, x[:, :1], x, table, lens)
    bad(cache, x, x[:3], table, lens)
    bad(cache, x[:3], x[:3], table, lens)                       # 3 rows of 2 sequences
    bad(cache, x.double(), x, table, lens)
    bad(cache, x[:, :, ::2], x, table, lens)
    bad(cache, x, x, table.long(), lens)
    bad(cache, x, x, table[0], lens)
    bad(cache, x, x, table, lens[:1])
    bad(cache, x, x, table, lens, ends=lens[:1])
    bad(cache, x.cpu(), x, table, lens)
    bad(cache, x, x, table, lens.cpu())
    with pytest.raises((ValueError, hatq.HatqError)):
        hatq.hatq_cache4_read(cache, 4, table, lens, k=x[:1].expand(4, 2, 64))      # rows that overlap
    for sizes in ((0, 16, 2, 64), (4, 8, 2, 64), (4, 24, 2, 64), (4, 16, 0, 64), (4, 16, 2, 257), (4, 16, 2, 0), (2 ** 31, 16, 2, 64)):
        with pytest.raises((ValueError, hatq.HatqError)):
            hatq.hatq_cache4_init(*sizes, device=DEV)
    with pytest.raises(hatq.HatqError):
        hatq.hatq_cache4_init(4, 16, 2, 96, hblock=64, device=DEV)
    with pytest.raises(hatq.HatqError) as e:
        hatq.hatq_cache4_init(4, 16, 2, 64, buf=torch.empty(100, dtype=torch.int8, device=DEV))
    assert e.value.status == hatq.HATQ_EWORKSPACE
    # no rows
    hatq.hatq_cache4_append(cache, x[:0], x[:0], table, lens)
    k, _ = hatq.hatq_cache4_read(cache, 0, table, lens)
    assert k.shape == (0, 2, 64)
