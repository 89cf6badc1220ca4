"""CPU-side checks of the C ABI of the linear layers of 4-bit weights: sizes, the struct's
layout, and the rejection of bad arguments on the host before any launch (fake pointers,
never dereferenced)."""
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


def weights(**over):
    w = hatq.Linear4Weights(4000, 100, 0, 8, 64, 4096, 112, P, P, P)
    for k, v in over.items():
        setattr(w, k, v)
    return w


def test_struct_layout():
    assert ctypes.sizeof(hatq.Linear4Weights) == 56 and hatq.Linear4Weights.wpack.offset == 32


def test_bytes(L):
    up = lambda v: (v + 255) // 256 * 256  # noqa: E731
    assert L.hatq_linear4_weights_bytes(1000, 100, 0, 8, 64) == up(112 * 512) + up(112 * 32) + up(112 * 4)
    assert L.hatq_linear4_weights_bytes(64, 17, 1, 64, 128) == up(64 * 64) + up(64 * 2) + up(64 * 4)
    assert L.hatq_linear4_weights_bytes(65536, 65536, 0, 128, 64) == 2 ** 31 + 2 ** 27 + 2 ** 18
    for bad in [(0, 16, 0, 1, 64), (64, 0, 0, 1, 64), (64, 16, 2, 1, 64), (64, 16, 0, 3, 64), (64, 16, 0, 0, 64), (64, 16, 0, 128, 64),
                (64, 16, 0, 1, 32), (64, 16, 0, 1, 0), (65537, 16, 0, 1, 64), (64, 65537, 0, 1, 64), (64, 32769, 1, 1, 64), (192, 16, 0, 192, 64)]:
        assert L.hatq_linear4_weights_bytes(*bad) == 0, bad
    w = weights()
    assert L.hatq_linear4_ws_bytes(ctypes.byref(w), 4) == 0
    assert L.hatq_linear4_ws_bytes(ctypes.byref(w), 5) == 16 * 4096 + 256
    assert L.hatq_linear4_ws_bytes(ctypes.byref(w), 2 ** 24) == (4096 << 24) + (4 << 24)
    wide = weights(cout=8208, cout_pad=8208)
    assert L.hatq_linear4_ws_bytes(ctypes.byref(wide), 2) == 0
    assert L.hatq_linear4_ws_bytes(ctypes.byref(wide), 3) == 16 * 4096 + 256
    short = weights(cin=1000, k_stride=1024)
    assert L.hatq_linear4_ws_bytes(ctypes.byref(short), 1000) == 0
    assert L.hatq_linear4_ws_bytes(ctypes.byref(short), 2 ** 24) == (1024 << 24) + (4 << 24)
    middle = weights(cin=2000, k_stride=2048)
    assert [L.hatq_linear4_ws_bytes(ctypes.byref(middle), n) for n in (3, 4, 65)] == [0, 16 * 2048 + 256, 0]
    for rows in (0, -1, 2 ** 24 + 1):
        assert L.hatq_linear4_ws_bytes(ctypes.byref(w), rows) == 0
    assert L.hatq_linear4_ws_bytes(None, 17) == 0
    assert L.hatq_linear4_ws_bytes(ctypes.byref(weights(k_stride=4032)), 17) == 0


@cpu_only
def test_weights_refusals(L):
    n = L.hatq_linear4_weights_bytes(1000, 100, 0, 8, 64)
    out = hatq.Linear4Weights()

    def prep(shape=(1000, 100, 0, 8, 64), w=P, t=0, bias=None, dst=P, size=n, o=out):
        return L.hatq_prepare_linear4(*shape, w, t, bias, dst, size, None if o is None else ctypes.byref(o), None)

    def pack(shape=(1000, 100, 0, 8, 64), codes=P, scale=P, bias=None, dst=P, size=n):
        return L.hatq_pack_linear4(*shape, codes, scale, bias, dst, size, ctypes.byref(out), None)
    for kw in (dict(w=None), dict(w=P + 2), dict(t=3), dict(t=1, w=P + 1), dict(bias=P + 2), dict(dst=None), dict(dst=P + 128), dict(o=None),
               dict(shape=(1000, 100, 0, 8, 32)), dict(shape=(1000, 100, 0, 5, 64))):
        assert prep(**kw) == EINVAL, kw
    for kw in (dict(codes=None), dict(scale=None), dict(scale=P + 1), dict(bias=P + 1), dict(dst=P + 1)):
        assert pack(**kw) == EINVAL, kw
    assert prep(size=n - 1) == EWORKSPACE and pack(size=n - 1) == EWORKSPACE
    assert prep(shape=(1000, 100, 0, 16, 64)) == EUNSUPPORTED and pack(shape=(960, 100, 0, 320, 64)) == EUNSUPPORTED


@cpu_only
def test_forward_refusals(L):
    def call(w=None, x=P, xt=0, rows=40, xs=4000, y=P, yt=0, ys=100, ws=P, size=2 ** 30):
        return L.hatq_linear4_forward(ctypes.byref(w or weights()), x, xt, rows, xs, y, yt, ys, ws, size, None)
    assert call(rows=0) == OK
    assert L.hatq_linear4_forward(None, P, 0, 40, 4000, P, 0, 100, P, 2 ** 30, None) == EINVAL
    for kw in (dict(x=None), dict(x=P + 1), dict(xt=3), dict(xs=3999), dict(xs=2 ** 60), dict(y=None), dict(y=P + 3), dict(yt=-1), dict(ys=99),
               dict(ws=None), dict(ws=P + 16), dict(rows=-1)):
        assert call(**kw) == EINVAL, kw
    for over in (dict(k_stride=4000), dict(cout_pad=100), dict(wpack=None), dict(wpack=P + 8), dict(w_scale=P + 2), dict(bias=None), dict(group=256),
                 dict(gated=1)):
        assert call(w=weights(**over)) == EINVAL, over
    assert call(size=40 * 4096 + 255) == EWORKSPACE
    assert call(rows=2 ** 24 + 1) == EUNSUPPORTED
