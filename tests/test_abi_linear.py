"""CPU-side checks of the linear layers' C ABI: sizes, layouts of the structs, and the
rejection of bad arguments on the host before any launch (fake pointers, never
dereferenced), also under AddressSanitizer and UndefinedBehaviorSanitizer."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_01653_amd import hatq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
P = 0x10000            # aligned to 256, never dereferenced

# Never where a GPU is visible: a validation bug would launch on garbage.
try:
    import torch
    _HAS_GPU = torch.cuda.device_count() > 0
except Exception:  # pragma: no cover
    _HAS_GPU = False
cpu_only = pytest.mark.skipif(_HAS_GPU, reason="fake-pointer validation tests run on CPU-only hosts")


@pytest.fixture(scope="module")
def L():
    return hatq.load(build_if_missing=True)


def weights(**over):
    w = hatq.LinearWeights(1, 192, 100, 0, 64, 192, 128, P, P, P)
    for k, v in over.items():
        setattr(w, k, v)
    return w


def test_weights_bytes(L):
    def size(e, cin, cout, gated, b):
        return L.hatq_linear_weights_bytes(e, cin, cout, gated, b)
    up = lambda v: (v + 255) // 256 * 256  # noqa: E731
    assert size(1, 192, 100, 0, 64) == up(128 * 192) + 2 * up(128 * 4)
    assert size(3, 65, 33, 1, 1) == up(3 * 128 * 128) + 2 * up(3 * 128 * 4)
    assert size(1024, 65536, 65536, 0, 128) == 1024 * 65536 * 65536 + 2 * 1024 * 65536 * 4
    for bad in [(0, 64, 16, 0, 1), (1, 0, 16, 0, 1), (1, 64, 0, 0, 1), (1, 64, 16, 2, 1), (1, 64, 16, 0, 3), (1, 64, 16, 0, 0),
                (1, 64, 16, 0, 128), (1, 192, 16, 0, 192), (1025, 64, 16, 0, 1), (1, 65537, 16, 0, 1), (1, 64, 32769, 1, 1),
                (1, 64, 65537, 0, 1), (1, 64, 16, 0, 256), (-1, 64, 16, 0, 1)]:
        assert size(*bad) == 0, bad


def test_ws_bytes(L):
    w = weights()
    assert L.hatq_linear_ws_bytes(ctypes.byref(w), 5) == 1024 + 256
    assert L.hatq_linear_ws_bytes(ctypes.byref(w), 1 << 24) == (192 << 24) + (4 << 24)
    for rows in (0, -1, (1 << 24) + 1):
        assert L.hatq_linear_ws_bytes(ctypes.byref(w), rows) == 0
    assert L.hatq_linear_ws_bytes(ctypes.byref(weights(k_stride=256)), 5) == 0
    assert L.hatq_linear_ws_bytes(None, 5) == 0
    assert L.hatq_expert_order_ws_bytes(0, 1, 1) > 0
    assert L.hatq_expert_order_ws_bytes(1 << 20, 16, 1024) > 0
    for bad in [(-1, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 1025), (1 << 20, 17, 4)]:
        assert L.hatq_expert_order_ws_bytes(*bad) == 0


@cpu_only
def test_refusals(L):
    EINVAL, UNSUP, EWS, OK = hatq.HATQ_EINVAL, hatq.HATQ_EUNSUPPORTED, hatq.HATQ_EWORKSPACE, hatq.HATQ_OK
    out = hatq.LinearWeights()
    n = 1 << 20
    prep = lambda *shape, w=P, t=0, b=None, dst=P, size=n, o=out: L.hatq_prepare_linear(  # noqa: E731
        *shape, w, t, b, dst, size, None if o is None else ctypes.byref(o), None)
    good = (1, 192, 100, 0, 64)
    assert prep(*good, w=None) == EINVAL
    assert prep(*good, t=3) == EINVAL
    assert prep(*good, w=P + 2) == EINVAL
    assert prep(*good, b=P + 1) == EINVAL
    assert prep(*good, dst=None) == EINVAL
    assert prep(*good, dst=P + 16) == EINVAL
    assert prep(*good, o=None) == EINVAL
    assert prep(*good, size=100) == EWS
    assert prep(1, 192, 100, 0, 48) == EINVAL
    assert prep(1, 192, 100, 0, 128) == UNSUP
    assert prep(1, 192, 100, 0, 192) == UNSUP
    assert prep(1, 1 << 30, 1 << 30, 0, 64) == UNSUP
    pack = lambda codes, s: L.hatq_pack_linear(*good, codes, s, None, P, n, ctypes.byref(out), None)  # noqa: E731
    assert pack(None, P) == EINVAL
    assert pack(P, None) == EINVAL
    assert pack(P, P + 2) == EINVAL
    assert bytes(out) == bytes(hatq.LinearWeights())       # untouched

    quant = lambda x=P, t=1, rows=4, cin=192, xs=192, b=64, xq=P, s=P: L.hatq_token_quant(  # noqa: E731
        x, t, rows, cin, xs, b, xq, s, None)
    assert quant(rows=0, x=None, xq=None, s=None) == OK
    for bad in [dict(x=None), dict(x=P + 1), dict(t=3), dict(t=-1), dict(rows=-1), dict(cin=0), dict(xs=191), dict(b=5),
                dict(xq=None), dict(xq=P + 8), dict(s=None), dict(s=P + 2), dict(xs=1 << 60)]:
        assert quant(**bad) == EINVAL, bad
    for bad in [dict(b=128), dict(b=320), dict(cin=1 << 17, xs=1 << 17), dict(rows=(1 << 24) + 1)]:
        assert quant(**bad) == UNSUP, bad

    def linear(w=None, xq=P, s=P, rows=4, y=P, t=0, ys=100):
        return L.hatq_linear_int8(ctypes.byref(w or weights()), xq, s, rows, y, t, ys, None)
    assert linear(rows=0, xq=None, y=None) == OK
    for bad in [dict(xq=None), dict(xq=P + 4), dict(s=None), dict(rows=-1), dict(y=None), dict(y=P + 2), dict(t=7), dict(ys=99),
                dict(w=weights(wpack=None)), dict(w=weights(wpack=P + 8)), dict(w=weights(cout_pad=100)),
                dict(w=weights(k_stride=128)), dict(w=weights(experts=2)), dict(w=weights(gated=2)), dict(w=weights(cin=0))]:
        assert linear(**bad) == EINVAL, bad
    assert linear(rows=(1 << 24) + 1) == UNSUP
    assert L.hatq_linear_int8(None, P, P, 4, P, 0, 100, None) == EINVAL

    def forward(w=None, x=P, t=1, rows=4, xs=192, y=P, yt=0, ys=100, ws=P, size=n):
        return L.hatq_linear_forward(ctypes.byref(w or weights()), x, t, rows, xs, y, yt, ys, ws, size, None)
    for bad in [dict(x=None), dict(xs=10), dict(t=9), dict(rows=17, ws=None), dict(rows=17, ws=P + 64), dict(ys=0)]:
        assert forward(**bad) == EINVAL, bad
    assert forward(rows=17, size=3583) == EWS
    wide = weights(cin=8192, k_stride=8192)
    assert forward(w=wide, rows=3, xs=8192, ws=None) == EINVAL
    assert forward(w=wide, rows=3, xs=8192, size=3 * 8192) == EWS

    def grouped(w=None, x_rows=3, ends=P, src=P, rows=8, y=P, ys=100, xq=P):
        return L.hatq_experts_int8(ctypes.byref(w or weights(experts=5)), xq, P, x_rows, ends, src, rows, y, 2, ys, None)
    assert grouped(rows=0, ends=None) == OK
    for bad in [dict(ends=None), dict(ends=P + 1), dict(src=P + 2), dict(src=None), dict(x_rows=0), dict(x_rows=-1), dict(y=None),
                dict(xq=None)]:
        assert grouped(**bad) == EINVAL, bad
    assert grouped(x_rows=(1 << 24) + 1) == UNSUP
    assert grouped(w=weights(experts=1025)) == UNSUP
    assert L.hatq_experts_forward(ctypes.byref(weights(experts=5)), P, 0, 3, 192, P, P, 8, P, 0, 100, P, 700, None) == EWS

    order = lambda ids=P, t=4, k=2, e=8, ends=P, src=P, pos=P, ws=P, size=n: L.hatq_expert_order(  # noqa: E731
        ids, t, k, e, ends, src, pos, ws, size, None)
    for bad in [dict(ids=None), dict(t=-1), dict(k=0), dict(e=0), dict(ends=None), dict(src=None), dict(pos=None), dict(ws=None),
                dict(ws=P + 4), dict(pos=P + 1)]:
        assert order(**bad) == EINVAL, bad
    assert order(e=1025) == UNSUP
    assert order(t=1 << 24, k=2) == UNSUP
    assert order(size=10) == EWS

    comb = lambda h=P, hr=8, c=64, hs=64, pos=P, w=P, t=4, k=2, y=P, yt=1, ys=64: L.hatq_expert_combine(  # noqa: E731
        h, hr, c, hs, pos, w, t, k, y, yt, ys, None)
    assert comb(t=0, h=None, y=None) == OK
    for bad in [dict(h=None), dict(hr=-1), dict(c=0), dict(hs=63), dict(pos=None), dict(w=None), dict(k=0), dict(t=-1), dict(y=None),
                dict(yt=5), dict(ys=1)]:
        assert comb(**bad) == EINVAL, bad


@cpu_only
def test_mlp_refusals(L):
    def mlp(w_in=None, w_out=None, x=P, t=1, n=4, xs=192, ids=P, w=P, k=2, y=P, yt=1, ys=192, ws=P, size=1 << 20):
        a, b = w_in or hatq.LinearWeights(5, 192, 64, 1, 64, 192, 128, P, P, P), w_out or hatq.LinearWeights(5, 64, 192, 0, 64, 64, 192, P, P, P)
        return L.hatq_expert_mlp(ctypes.byref(a), ctypes.byref(b), x, t, n, xs, ids, w, k, y, yt, ys, ws, size, None)
    assert mlp(n=0, x=None) == hatq.HATQ_OK
    plain = hatq.LinearWeights(5, 192, 64, 0, 64, 192, 64, P, P, P)
    other = hatq.LinearWeights(4, 64, 192, 0, 64, 64, 192, P, P, P)
    wide = hatq.LinearWeights(5, 128, 192, 0, 64, 128, 192, P, P, P)
    for bad in [dict(w_in=plain), dict(w_out=other), dict(w_out=wide), dict(x=None), dict(n=-1), dict(k=0), dict(xs=1), dict(ids=None),
                dict(w=None), dict(w=P + 2), dict(y=None), dict(ys=5), dict(t=4), dict(ws=None), dict(ws=P + 32)]:
        assert mlp(**bad) == hatq.HATQ_EINVAL, bad
    assert mlp(size=100) == hatq.HATQ_EWORKSPACE
    assert mlp(n=1 << 23, k=4) == hatq.HATQ_EUNSUPPORTED


DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include "hatq.h"
#include "linear.h"
namespace hatq {   // no launch may be reached
hipError_t launch_token_quant(const TokenArgs &, hipStream_t) { std::abort(); }
hipError_t launch_linear_prepare(const LinearPrepArgs &, hipStream_t) { std::abort(); }
hipError_t launch_linear(const LinearArgs &, hipStream_t) { std::abort(); }
bool linear_takes_tokens(const LinearArgs &a) { return a.rows & 1; }
hipError_t launch_linear_tokens(const LinearArgs &, const TokenArgs &, hipStream_t) { std::abort(); }
hipError_t launch_expert_order(const OrderArgs &, hipStream_t) { std::abort(); }
hipError_t launch_expert_combine(const CombineArgs &, hipStream_t) { std::abort(); }
hipError_t launch_order_quant(const OrderArgs &, const TokenArgs &, hipStream_t) { std::abort(); }
size_t expert_order_ws_ints(int64_t pairs, int32_t experts) { return (size_t)pairs * experts; }
}
int main() {
    void *const F = reinterpret_cast<void *>(0x10000);
    auto *b = static_cast<int8_t *>(F);
    auto *f = static_cast<float *>(F);
    auto *i = static_cast<int32_t *>(F);
    const int32_t ends[] = {INT32_MIN, -1, 0, 1, 3, 64, 192, 320, 1024, 65536, 1 << 24, INT32_MAX};
    // every extreme of every size: rejected (a null or a small buffer sees to the rest)
    for (int32_t a : ends)
        for (int32_t c : ends)
            for (int32_t d : ends) {
                (void)hatq_linear_weights_bytes(a, c, d, a & 1, 64);
                (void)hatq_linear_weights_bytes(a, c, d, 1, 1);
                (void)hatq_expert_order_ws_bytes(a, c, d);
                hatq_linear_weights W{}, o{};
                W = {a, c, d, 0, 1, c > 0 && c < 1 << 20 ? (c + 63) / 64 * 64 : c, d > 0 && d < 1 << 20 ? (d + 31) / 32 * 32 : d, b, f, f};
                for (int32_t rows : ends) {
                    (void)hatq_linear_ws_bytes(&W, rows);
                    if (rows == 0) continue;
                    if (!hatq_linear_int8(&W, nullptr, f, rows, F, 0, (int64_t)d, nullptr)) return 1;
                    if (!hatq_linear_forward(&W, F, 0, rows, INT64_MAX, F, 0, INT64_MAX, F, 1, nullptr)) return 2;
                    if (!hatq_experts_forward(&W, F, 1, rows, c, i, i, rows, F, 0, d, F, 1, nullptr)) return 3;
                    if (!hatq_token_quant(F, 0, rows, c, INT64_MAX, 1, b, f, nullptr)) return 4;
                }
                hatq_linear_weights G = W;
                G.gated = 1;
                (void)hatq_expert_mlp_ws_bytes(&G, &W, c, d);
                if (a > 0 && !hatq_expert_mlp(&G, &W, F, 0, a, c, i, f, d, F, 0, d, F, 1, nullptr)) return 9;
                if (!hatq_prepare_linear(a, c, d, 0, 1, F, 0, nullptr, F, 1, &o, nullptr)) return 5;
                if (!hatq_pack_linear(a, c, d, 1, 1, b, f, nullptr, F, 1, &o, nullptr)) return 6;
                if (!hatq_expert_order(i, a, c, d, i, i, i, F, 1, nullptr)) return 7;
                if (a != 0 && !hatq_expert_combine(f, c, d, INT64_MAX, i, nullptr, a, 1, F, 0, INT64_MAX, nullptr)) return 8;
            }
    std::puts("ok");
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(f"{ROCM}/include/hip/hip_runtime.h"),
                    reason="needs g++ and the HIP headers")
def test_validation_sanitized(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    csrc = f"{ROOT}/paper_2608_01653_amd/csrc"
    exe = str(tmp_path / "san")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{ROOT}/include", f"-I{csrc}",
                    "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-O1", "-g", f"{csrc}/api_linear.cpp",
                    str(tmp_path / "driver.cpp"), f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib", "-o", exe],
                   check=True, capture_output=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout + r.stderr
