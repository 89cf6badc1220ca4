"""CPU-side checks of the C ABI of the 4-bit cache and the attention over it: sizes, layouts
of the structs, and the rejection of bad arguments on the host before any launch (fake
pointers, never dereferenced)."""
import ctypes

import pytest

from paper_2608_01653_amd import hatq

P = 0x10000            # aligned to 256, never dereferenced

# Never where a GPU is visible: a validation bug would launch on garbage.
try:
    import torch
    _HAS_GPU = torch.cuda.device_count() > 0
except Exception:  # pragma: no cover
    _HAS_GPU = False
cpu_only = pytest.mark.skipif(_HAS_GPU, reason="fake-pointer validation tests run on CPU-only hosts")
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = (hatq.HATQ_OK, hatq.HATQ_EINVAL, hatq.HATQ_EUNSUPPORTED, hatq.HATQ_EWORKSPACE)


@pytest.fixture(scope="module")
def L():
    return hatq.load(build_if_missing=True)


def cache(**over):
    c = hatq.Cache4View(10, 64, 4, 128, 64, P)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def heads(**over):
    x = hatq.Heads(1, 512, 128, P)
    for k, v in over.items():
        setattr(x, k, v)
    return x


def test_struct_layouts():
    assert ctypes.sizeof(hatq.Cache4View) == 32 and hatq.Cache4View.buf.offset == 24
    assert ctypes.sizeof(hatq.Heads) == 32 and hatq.Heads.p.offset == 24


def test_bytes(L):
    assert L.hatq_cache4_bytes(10, 64, 4, 128, 64) == 10 * 64 * 4 * 2 * 68
    assert L.hatq_cache4_bytes(3, 16, 1, 1, 1) == 3 * 16 * 68
    assert L.hatq_cache4_bytes(2 ** 15, 2 ** 15, 1024, 256, 128) == 2 ** 30 * 1024 * 4 * 68
    for bad in [(0, 64, 4, 128, 64), (10, 8, 4, 128, 64), (10, 48, 4, 128, 64), (10, 2 ** 17, 4, 128, 64), (10, 64, 0, 128, 64),
                (10, 64, 4, 0, 1), (10, 64, 4, 257, 1), (10, 64, 4, 128, 3), (10, 64, 4, 128, 0), (10, 64, 4, 96, 64), (10, 64, 4, 192, 192),
                (10, 64, 1025, 128, 64), (2 ** 16, 2 ** 16, 1, 64, 1), (-1, 64, 4, 128, 64), (10, -64, 4, 128, 64), (10, 64, 4, 256, 256)]:
        assert L.hatq_cache4_bytes(*bad) == 0, bad


def test_init(L):
    out = hatq.Cache4View()
    n = L.hatq_cache4_bytes(10, 64, 4, 128, 64)
    ref = ctypes.byref(out)
    assert L.hatq_cache4_init(10, 64, 4, 128, 64, P, n, ref) == OK
    assert (out.pages, out.page_size, out.heads, out.dim, out.hblock, out.buf) == (10, 64, 4, 128, 64, P)
    assert L.hatq_cache4_init(10, 64, 4, 128, 64, P, n - 1, ref) == EWORKSPACE
    assert L.hatq_cache4_init(10, 64, 4, 128, 64, P + 128, n, ref) == EINVAL
    assert L.hatq_cache4_init(10, 64, 4, 128, 64, None, n, ref) == EINVAL
    assert L.hatq_cache4_init(10, 64, 4, 128, 64, P, n, None) == EINVAL
    assert L.hatq_cache4_init(10, 64, 4, 128, 192, P, n, ref) == EUNSUPPORTED


def cache_call(L, which, c, k, v, rows=8, table=P, width=3, lens=P, ends=None, batch=4):
    call = L.hatq_cache4_append if which == "append" else L.hatq_cache4_read
    by = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return call(by(c), by(k), by(v), rows, table, width, lens, ends, batch, None)


@cpu_only
@pytest.mark.parametrize("which", ["append", "read"])
def test_cache_refusals(L, which):
    def call(c=None, k=None, v=None, **kw):
        return cache_call(L, which, c or cache(), k or heads(), v or heads(), **kw)
    assert call(rows=0) == OK
    assert cache_call(L, which, None, heads(), heads()) == EINVAL
    assert cache_call(L, which, cache(), None, heads()) == EINVAL
    assert cache_call(L, which, cache(), heads(), None) == EINVAL
    for over in (dict(pages=0), dict(page_size=24), dict(heads=0), dict(dim=0), dict(hblock=5), dict(buf=None), dict(buf=P + 16)):
        assert call(c=cache(**over)) == EINVAL, over
    for over in (dict(hblock=192), dict(dim=300), dict(heads=2000), dict(pages=2 ** 27)):
        assert call(c=cache(**over)) == EUNSUPPORTED, over
    for over in (dict(type=3), dict(type=-1), dict(p=None), dict(p=P + 1), dict(row_stride=-1), dict(head_stride=-1), dict(row_stride=2 ** 62),
                 dict(head_stride=2 ** 62), dict(type=0, p=P + 2)):
        assert call(k=heads(**over)) == EINVAL, over
        assert call(v=heads(**over)) == EINVAL, over
    for kw in (dict(rows=-1), dict(rows=7), dict(width=0), dict(batch=0), dict(batch=-2), dict(table=None), dict(lens=None), dict(table=P + 2),
               dict(lens=P + 1), dict(ends=P + 2)):
        assert call(**kw) == EINVAL, kw
    assert call(rows=2 ** 24 + 4) == EUNSUPPORTED
    assert call(width=2 ** 24 + 1) == EUNSUPPORTED


@cpu_only
def test_outputs_that_overlap(L):
    for over in (dict(row_stride=511), dict(head_stride=127), dict(row_stride=0), dict(head_stride=0), dict(row_stride=128, head_stride=8 * 128 - 1 - 128)):
        assert cache_call(L, "read", cache(), heads(**over), heads()) == EINVAL, over


def attend(L, c=None, q=None, y=None, rows=8, q_heads=8, table=P, width=3, lens=P, ends=None, batch=4, scale=0.1, causal=1, window=0, max_len=0,
           ws=P, ws_bytes=2 ** 40):
    by = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    wide = heads(row_stride=1024)
    return L.hatq_attention4(by(c or cache()), by(q or wide), by(y or wide), rows, q_heads, table, width, lens, ends, batch, scale, causal, window,
                             max_len, ws, ws_bytes, None)


@cpu_only
def test_attention_refusals(L):
    assert attend(L, rows=0) == OK
    wide = dict(row_stride=1024)
    for over in (dict(type=5), dict(p=None), dict(p=P + 1), dict(row_stride=-1)):
        assert attend(L, q=heads(**{**wide, **over})) == EINVAL, over
    for over in (dict(type=5), dict(p=None), dict(p=P + 1), dict(row_stride=512), dict(head_stride=100)):
        assert attend(L, y=heads(**{**wide, **over})) == EINVAL, over
    for kw in (dict(q_heads=7), dict(q_heads=0), dict(q_heads=-4), dict(rows=-8), dict(rows=9), dict(table=None), dict(lens=None), dict(ends=P + 1),
               dict(batch=0), dict(width=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(causal=-1), dict(window=-1),
               dict(window=3, causal=0), dict(max_len=-1)):
        assert attend(L, **kw) == EINVAL, kw
    for kw in (dict(q_heads=2 ** 14 + 4), dict(rows=2 ** 24 + 4), dict(width=2 ** 25), dict(rows=2 ** 24, q_heads=128)):
        assert attend(L, **kw) == EUNSUPPORTED, kw
    # a long table: the positions are split, and need a workspace
    kw = dict(width=4096)
    need = L.hatq_attention4_ws_bytes(ctypes.byref(cache()), 8, 8, 4096, 4, 0, 0, 0)
    assert need > 0
    assert attend(L, **kw, ws=None) == EINVAL
    assert attend(L, **kw, ws=P + 128) == EINVAL
    assert attend(L, **kw, ws_bytes=need - 1) == EWORKSPACE


def test_workspace_bytes(L):
    def size(c, *a):
        return L.hatq_attention4_ws_bytes(ctypes.byref(c), *a)
    assert size(cache(), 0, 8, 4096, 4, 0, 0, 0) == 0
    assert size(cache(), 8, 8, 1, 4, 0, 0, 0) == 0
    assert size(cache(), 8, 8, 4096, 4, 0, 0, 32) == 0
    assert size(cache(), 8, 7, 4096, 4, 0, 0, 0) == 0
    assert L.hatq_attention4_ws_bytes(None, 8, 8, 4096, 4, 0, 0, 0) == 0
    # as many parts as fit, none larger than the other: bounded however long the table
    assert size(cache(), 1, 4, 2 ** 24, 1, 0, 0, 0) <= 2 ** 26
