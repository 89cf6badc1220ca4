"""Linear layers of 4-bit weights against a plain implementation in 64 bits, over rows from
one to many, odd widths, both groups, gates, biases, types and strides.

Tolerances, derived from the arithmetic (u = 2^-24): the token's codes and scale are bit-exact
against the same float32 arithmetic in numpy; a group's sum is exact, and so is its float32
value (below 2^24 over 16, a multiple of 16).  n groups are summed in float32 by fma in some
order, n u of the sum of magnitudes A = sum |w_scale sum q wq| (each partial sum rounds
once), and the factor s / b and the bias add 2 u each: |z - z64| <= ((n + 8) A s / b + 2
(|z| + |bias|)) u.  A gated layer: |silu'| < 1.1, so an error d of the gate moves y by at
most 1.1 |u_| d and one of the value by |silu(g)| d; the unit itself adds 8 u |y|."""
import numpy as np
import pytest
import torch

from cache4_util import ROUND, U, butterfly, check, to_bf16
from gpu_util import DEV, Guarded, dev, host
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def token_codes(x, b):
    """(codes, scales fp32) of fp32 tokens, the kernel's arithmetic in numpy."""
    with np.errstate(all="ignore"):
        s = butterfly(x.astype(np.float32), b)
        most = np.abs(s).max(axis=1)
        scale = (most / np.float32(127.0)).astype(np.float32)
        scale[scale == 0] = 1.0
        q = np.clip(np.rint(s / scale[:, None]), -127, 127)
        bad = ~np.isfinite(most)
        scale[bad] = np.nan
        q[bad] = 0
    return q.astype(np.float64), scale.astype(np.float64)


def layer64(x, codes, w_scale, bias, b, group, gated):
    """(y, bound) in 64 bits; w_scale float64 [held, groups]."""
    q, s = token_codes(x, b)
    cin, n = x.shape[1], w_scale.shape[1]
    z, mag = np.zeros((x.shape[0], codes.shape[0])), np.zeros((x.shape[0], codes.shape[0]))
    for g in range(n):
        part = (q[:, g * group:(g + 1) * group] @ codes[:, g * group:(g + 1) * group].T.astype(np.float64)) * w_scale[:, g]
        z += part
        mag += np.abs(part)
    f = s[:, None] / b
    z, mag = z * f, mag * f
    bias = np.zeros(codes.shape[0]) if bias is None else bias
    z = z + bias
    err = ((n + 8) * mag + 2 * (np.abs(z) + np.abs(bias))) * U
    if not gated:
        return z, err
    half = codes.shape[0] // 2
    g, u = z[:, :half], z[:, half:]
    silu = g / (1 + np.exp(-g))
    y = silu * u
    return y, 1.1 * np.abs(u) * err[:, :half] + (np.abs(silu) + 1.1 * err[:, :half]) * err[:, half:] + 8 * U * np.abs(y)


def layer(rng, held, cin, group, bias):
    codes = rng.integers(-8, 8, size=(held, cin)).astype(np.int8)
    scale = to_bf16(rng.uniform(0.5, 1.5, size=(held, -(-cin // group))) / np.sqrt(cin))
    return codes, scale, rng.normal(size=held).astype(np.float32) if bias else None


def tokens(rng, rows, cin, dtype):
    x = rng.normal(size=(rows, cin)) * np.exp(0.5 * rng.normal(size=cin))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def packed(codes, scale, bias, hblock, gated):
    return hatq.hatq_pack_linear4(dev(codes), dev(scale).to(torch.bfloat16), bias=None if bias is None else dev(bias),
                                  hblock=hblock, gated=gated)


def compare(x, y, codes, scale, bias, hblock, group, gated, what=""):
    y64, bound = layer64(x.float().cpu().numpy(), codes, scale.astype(np.float64), bias, hblock, group, gated)
    check(y, y64, bound, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("rows,cin,cout,hblock", [(1, 512, 64, 128), (1, 4096, 16, 64), (3, 64, 17, 64), (16, 1000, 33, 8), (1, 8192, 40, 1),
                                                  (2, 8192, 16, 128), (1, 16384, 18, 128), (1, 1, 1, 1), (5, 65, 15, 1), (16, 1024, 100, 32),
                                                  (17, 512, 50, 64), (6, 4096, 70, 128), (33, 129, 31, 1), (64, 640, 48, 128), (65, 200, 9, 8), (9, 2176, 33, 128), (20, 2200, 97, 8), (40, 2304, 65, 64),
                                                  (130, 384, 257, 128), (3, 8320, 20, 64), (300, 100, 40, 4), (1, 20480, 24, 64)])
def test_against_64_bits(rows, cin, cout, hblock, group, gated, dtype):
    rng = np.random.default_rng(rows * cin + cout)
    held = 2 * cout if gated else cout
    codes, scale, bias = layer(rng, held, cin, group, rows % 2 == 1)
    if -(-cin // 64) == -(-cin // 128):
        group = 128
    x = tokens(rng, rows, cin, dtype)
    lin = packed(codes, scale, bias, hblock, gated)
    assert lin.group == group
    y = hatq.hatq_linear4_forward(lin, x.to(DEV))
    compare(x, y, codes, scale, bias, hblock, group, gated, f"{rows} x {cin} -> {cout}")
    assert torch.equal(y, hatq.hatq_linear4_forward(lin, x.to(DEV)))


@pytest.mark.parametrize("w_type", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("cin,cout,hblock,group", [(256, 33, 128, 64), (100, 20, 4, 128), (192, 16, 64, 128), (1, 3, 1, 64)])
def test_prepared_weights(cin, cout, hblock, group, gated, w_type):
    """Codes and scales of float weights, seen through rows of the identity: the outputs of
    unit codes are the weights' values."""
    rng = np.random.default_rng(cin)
    held = 2 * cout if gated else cout
    w = torch.from_numpy((rng.normal(size=(held, cin)) * np.exp(rng.normal(size=(held, 1)))).astype(np.float32)).to(w_type)
    w[min(5, held - 1)] = 0
    bias = rng.normal(size=held).astype(np.float32)
    lin = hatq.hatq_prepare_linear4(w.to(DEV), dev(bias), hblock=hblock, group=group, gated=gated)
    t = butterfly(w.double().numpy(), hblock).astype(np.float32)
    codes, scale = np.zeros((held, cin), np.int8), np.zeros((held, -(-cin // group)), np.float32)
    for g in range(scale.shape[1]):
        part = t[:, g * group:(g + 1) * group]
        s = np.maximum(to_bf16((np.abs(part).max(1) / np.float32(7)).astype(np.float32)), np.float32(2.0 ** -100))
        scale[:, g] = s
        codes[:, g * group:(g + 1) * group] = np.clip(np.rint(part / s[:, None]), -7, 7)
    x = tokens(rng, 9, cin, torch.float32)
    compare(x, hatq.hatq_linear4_forward(lin, x.to(DEV)), codes, scale, bias, hblock, group, gated)
    # the very codes: the layer packed from them gives the same bits
    other = packed(codes, scale, bias, hblock, gated)
    if other.group == group:
        assert torch.equal(hatq.hatq_linear4_forward(lin, x.to(DEV)), hatq.hatq_linear4_forward(other, x.to(DEV)))


def test_codes_outside_are_taken_in():
    rng = np.random.default_rng(3)
    codes, scale, _ = layer(rng, 20, 128, 64, False)
    wild = codes.copy()
    wild[codes == 7] = 100
    wild[codes == -8] = -128
    a, b = packed(codes, scale, None, 64, False), packed(wild, scale, None, 64, False)
    x = tokens(rng, 4, 128, torch.float32).to(DEV)
    assert torch.equal(hatq.hatq_linear4_forward(a, x), hatq.hatq_linear4_forward(b, x))


@pytest.mark.parametrize("rows", [3, 40])
def test_not_finite(rows):
    """A token that is not finite: its row is NaN, no other; a scale that is NaN: its channel."""
    rng = np.random.default_rng(rows)
    codes, scale, bias = layer(rng, 40, 256, 64, True)
    scale[11, 2] = np.nan
    lin = packed(codes, scale, bias, 64, False)
    x = tokens(rng, rows, 256, torch.float32)
    x[1, 100] = float("inf")
    y = host(hatq.hatq_linear4_forward(lin, x.to(DEV)))
    want = np.zeros(y.shape, bool)
    want[1], want[:, 11] = True, True
    assert (np.isnan(y) == want).all()
    # float weights: a group that is not finite
    w = rng.normal(size=(20, 256)).astype(np.float32)
    w[7, 130] = np.inf
    y = host(hatq.hatq_linear4_forward(hatq.hatq_prepare_linear4(dev(w), hblock=64, group=64), x[2:3].to(DEV)))
    assert (np.isnan(y)[0] == (np.arange(20) == 7)).all()


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.float32), (torch.float32, torch.float16), (torch.float16, torch.bfloat16)])
@pytest.mark.parametrize("rows,cin", [(1, 200), (5, 200), (70, 200), (9, 2056), (40, 2200)])
def test_strides_and_types(rows, cin, dtype, out):
    rng = np.random.default_rng(rows)
    codes, scale, bias = layer(rng, 37, cin, 128, True)
    lin = packed(codes, scale, bias, 8, False)
    x = tokens(rng, rows, cin, dtype)
    wide = torch.zeros((rows, cin + 11), dtype=dtype, device=DEV)
    wide[:, 7:7 + cin] = x.to(DEV)
    y = torch.full((rows, 45), 3.0, dtype=out, device=DEV)
    ws = Guarded((max(256, hatq.hatq_linear4_ws_bytes(lin, rows)),), torch.int8)
    hatq.hatq_linear4_forward(lin, wide[:, 7:7 + cin], y=y[:, 5:42], ws=ws.view)
    ws.check("workspace")
    compare(x, y[:, 5:42], codes, scale, bias, 8, 128, False)
    assert bool((y[:, :5] == 3).all()) and bool((y[:, 42:] == 3).all())


def test_captured_and_replayed():
    rng = np.random.default_rng(5)
    codes, scale, bias = layer(rng, 64, 512, 64, True)
    lin = packed(codes, scale, bias, 64, True)
    long = packed(*layer(rng, 64, 2240, 64, True), 64, True)
    for rows, lin in ((2, lin), (40, lin), (40, long)):
        cin = lin.cin
        x = torch.zeros((rows, cin), dtype=torch.bfloat16, device=DEV)
        y = torch.zeros((rows, 32), dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(max(256, hatq.hatq_linear4_ws_bytes(lin, rows)), dtype=torch.int8, device=DEV)
        hatq.hatq_linear4_forward(lin, x, y=y, ws=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hatq.hatq_linear4_forward(lin, x, y=y, ws=ws)
        for _ in range(3):
            x.copy_(torch.randn((rows, cin)))
            graph.replay()
            eager = hatq.hatq_linear4_forward(lin, x)
            torch.cuda.synchronize()
            assert torch.equal(y, eager)


def test_refusals():
    rng = np.random.default_rng(6)
    codes, scale, bias = layer(rng, 32, 256, 64, True)
    lin = packed(codes, scale, bias, 64, False)
    x = torch.zeros((20, 256), device=DEV)

    def bad(f, *a, **k):
        with pytest.raises((ValueError, hatq.HatqError)):
            f(*a, **k)
    bad(hatq.hatq_linear4_forward, lin, x[:, :255])
    bad(hatq.hatq_linear4_forward, lin, x.double())
    bad(hatq.hatq_linear4_forward, lin, x.cpu())
    bad(hatq.hatq_linear4_forward, lin, x, y=torch.zeros((20, 33), device=DEV))
    bad(hatq.hatq_linear4_forward, lin, x, y=torch.zeros((1, 32), device=DEV).expand(20, 32))
    long = packed(*layer(rng, 32, 2176, 128, False), 64, False)
    bad(hatq.hatq_linear4_forward, long, torch.zeros((20, 2176), device=DEV), ws=torch.empty(256, dtype=torch.int8, device=DEV))
    bad(hatq.hatq_linear4_forward, lin, x, out_dtype=torch.int8)
    s = dev(scale).to(torch.bfloat16)
    bad(hatq.hatq_pack_linear4, dev(codes).float(), s)
    bad(hatq.hatq_pack_linear4, dev(codes), s.float())
    bad(hatq.hatq_pack_linear4, dev(codes), s[:, :3])
    bad(hatq.hatq_pack_linear4, dev(codes), s[:31])
    bad(hatq.hatq_pack_linear4, dev(codes[:31]), s[:31], gated=True)
    bad(hatq.hatq_pack_linear4, dev(codes), s, bias=dev(bias[:31]))
    bad(hatq.hatq_pack_linear4, dev(codes), s, hblock=3)
    bad(hatq.hatq_pack_linear4, dev(codes[:, :200]), s, hblock=64)
    bad(hatq.hatq_prepare_linear4, x, group=32)
    bad(hatq.hatq_prepare_linear4, x, hblock=192)
    assert hatq.hatq_linear4_forward(lin, x[:0]).shape == (0, 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cin,cout", [(1, 600, 20), (3, 2048, 33), (4, 2048, 33), (1, 1000, 8200), (2, 4096, 8200), (3, 4096, 8200), (4, 4000, 8192),
                                           (3, 2048, 8200), (70, 1504, 40), (90, 2048, 33)])
def test_few_rows(rows, cin, cout, gated, dtype):
    """The sizes at which rows change kernels."""
    rng = np.random.default_rng(rows + cin + cout)
    codes, scale, bias = layer(rng, cout * (2 if gated else 1), cin, 64, True)
    x = tokens(rng, rows, cin, dtype)
    y = hatq.hatq_linear4_forward(packed(codes, scale, bias, 8, gated), x.to(DEV))
    compare(x, y, codes, scale, bias, 8, 64, gated)


@pytest.mark.parametrize("rows,gated", [(12, False), (30, False), (100, False), (12, True), (20, True), (100, True)])
def test_many_groups(rows, gated):
    """Channels enough for waves that take several groups of them, and one group past the last
    whole set; the reference in float64 on the GPU."""
    rng = np.random.default_rng(rows)
    cin, cout, group = 2176, 16 * 1025 - 3, 64
    held = cout * (2 if gated else 1)
    codes, scale, bias = layer(rng, held, cin, group, True)
    x = tokens(rng, rows, cin, torch.float32)
    y = hatq.hatq_linear4_forward(packed(codes, scale, bias, 64, gated), x.to(DEV))
    compare(x, y, codes, scale, bias, 64, group, gated)
