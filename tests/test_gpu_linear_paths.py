"""Every kernel of the linear layers over tokens in every form (one layer or by expert,
plain or gated), at odd sizes: test_linear_choice.py shows on the CPU that these shapes
meet them all.

The sums stay below 2^24 and the scales are powers of two, so a plain layer's fp32 outputs
are the numbers themselves and 16-bit ones are these rounded once.  Gated outputs are
within 8 u |y| of 64 bits (u = 2^-24; the bound of test_gpu_linear_gate.py, z being exact).
Floats in give the bits of the two steps one after the other.
"""
import numpy as np
import pytest
import torch

from gpu_util import DEV, Guarded, dev
from paper_2608_01653_amd import hatq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# (rows, cin, cout, experts or 0 for one layer, gated) of codes: contractions of one step of
# 64 bytes, of fewer steps than a ring has buffers, of odd lengths and long ones
PRODUCTS = [
    # 16 rows streamed, by 2, 4 and 8 waves a group of channels
    (4084, 32, 19, 0, 0), (2193, 335, 49, 0, 0), (2937, 32, 35, 0, 1), (1377, 333, 81, 0, 1), (3746, 31, 34, 4, 0), (2703, 341, 39, 11, 0),
    (4196, 34, 21, 18, 1), (1303, 371, 87, 8, 1), (2451, 30, 17, 0, 0), (1387, 335, 35, 0, 0), (2253, 31, 17, 0, 1), (1367, 337, 37, 0, 1),
    (2246, 30, 21, 3, 0), (1001, 349, 53, 3, 0), (2018, 31, 18, 8, 1), (1121, 349, 53, 4, 1), (2, 30, 8, 0, 0), (1, 345, 33, 0, 0),
    (1, 30, 8, 0, 1), (1, 339, 33, 0, 1), (1, 31, 10, 1, 0), (1, 385, 33, 3, 0), (1, 33, 8, 1, 1), (1, 333, 33, 3, 1),
    # 32 rows streamed
    (17, 555, 8988, 0, 0), (4099, 495, 67, 0, 0), (18, 266, 7914, 0, 1), (19, 333, 6225, 0, 1), (5475, 854, 16, 260, 0), (2777, 781, 53, 166, 0),
    (2655, 1102, 8, 204, 1), (1849, 689, 37, 118, 1), (18, 4529, 13060, 0, 0),
    # tiles of 32 x 64 and 64 x 64, the contraction over four groups of waves
    (4887, 34, 8, 0, 0), (4123, 335, 33, 0, 0), (4287, 31, 9, 0, 1), (1975, 431, 33, 0, 1), (4186, 33, 10, 1, 0), (4237, 359, 37, 5, 0),
    (4964, 35, 8, 2, 1), (2221, 405, 41, 4, 1), (9298, 139, 8, 0, 0), (4155, 365, 65, 0, 0), (8510, 155, 8, 0, 1), (4275, 335, 33, 0, 1),
    (11153, 139, 9, 4, 0), (10063, 343, 35, 7, 0), (11691, 130, 10, 4, 1), (4515, 367, 33, 25, 1),
    # 64 x 128, 128 x 128, 128 x 256
    (6581, 31, 9, 0, 0), (8309, 359, 65, 0, 0), (7239, 33, 8, 0, 1), (8389, 367, 35, 0, 1), (7216, 32, 9, 19, 0), (8427, 387, 73, 3, 0),
    (6494, 41, 10, 1, 1), (8357, 339, 33, 23, 1), (8207, 731, 130, 0, 0), (8199, 713, 133, 0, 0), (8319, 647, 78, 0, 1), (8707, 671, 67, 0, 1),
    (9289, 2735, 134, 6, 0), (9451, 2413, 137, 5, 0), (11707, 2272, 74, 21, 1), (8771, 2785, 65, 8, 1), (5581, 65, 4134, 0, 0),
    (6621, 395, 519, 0, 0), (8030, 31, 3012, 0, 1), (8633, 385, 205, 0, 1), (8680, 76, 2869, 1, 0), (9703, 587, 415, 7, 0),
    (7121, 71, 1608, 1, 1), (10771, 533, 199, 5, 1), (2721, 534, 1813, 3, 1),
    # 256 x 256, four buffers
    (3974, 1158, 3159, 0, 0), (8389, 1155, 1439, 0, 0), (2305, 4096, 4100, 0, 0), (6186, 1159, 989, 0, 1), (5271, 1099, 1163, 0, 1),
    (7065, 7364, 2013, 1, 0), (10297, 8845, 1041, 4, 0), (7473, 7978, 861, 2, 1), (11833, 3889, 1183, 4, 1),
]

# and of floats: the small kernel with 1, 2 and 4 chunks a lane, by expert too, and several
# ranges of columns; the few-token kernel; tokens that are quantized first
FORWARDS = [
    (301, 320, 201, 0, 0), (6001, 192, 70, 0, 1), (77, 1000, 101, 0, 0), (333, 960, 300, 0, 1), (701, 1900, 130, 0, 0), (701, 1900, 500, 0, 0),
    (601, 2048, 70, 0, 1), (601, 2048, 301, 0, 1), (300, 128, 16, 16, 0), (96, 512, 48, 32, 1), (96, 1000, 70, 32, 0), (51, 1024, 300, 9, 1),
    (48, 2048, 300, 64, 0), (77, 1930, 140, 12, 1), (3, 1900, 45, 0, 0), (4, 4096, 64, 0, 1), (2, 8000, 33, 0, 0), (2, 8192, 49, 0, 1),
    (1, 16384, 40, 0, 0), (1, 12288, 70, 0, 1), (40, 4096, 130, 0, 0), (901, 4160, 130, 5, 1)]


def ragged(rng, e, rows):
    """Row ends of e experts, some without a row, a few rows past the last end."""
    return np.cumsum(rng.multinomial(rows - min(rows // 4, 7), rng.dirichlet(np.full(e, 0.5)))).astype(np.int32)


def sources(rng, rows, x_rows):
    src = rng.integers(0, x_rows, rows).astype(np.int32)
    if rows > 8:
        src[rng.integers(0, rows, 4)] = (-1, x_rows, 2 ** 31 - 1, -2 ** 31)
    return src


@pytest.mark.parametrize("rows,cin,cout,e,gated", PRODUCTS)
def test_codes(rows, cin, cout, e, gated):
    rng = np.random.default_rng(rows + cin)
    gen = torch.Generator(device=DEV).manual_seed(rows)
    held, experts = cout * (1 + gated), max(e, 1)
    lim = min(127, max(1, int((2 ** 24 / cin) ** 0.5) - 1))
    codes = torch.randint(-lim, lim + 1, (experts, held, cin), generator=gen, device=DEV).to(torch.int8)
    bias = torch.randint(-8, 9, (experts, held), generator=gen, device=DEV).float()
    step = 2.0 ** -18 if gated else 1.0
    lin = hatq.hatq_pack_linear(codes, torch.full((experts, held), step, device=DEV), bias * step, gated=bool(gated))
    x_rows = rows // 2 + 1 if e else rows
    q = torch.zeros((x_rows, lin.k_stride), dtype=torch.int8, device=DEV)
    q[:, :cin] = torch.randint(-lim, lim + 1, (x_rows, cin), generator=gen, device=DEV)
    ends = ragged(rng, e, rows) if e else np.array([rows])
    src = sources(rng, rows, x_rows) if e else np.arange(rows)

    # z in 64 bits: whole numbers below 2^24, times `step`; 0 past the last end
    z = torch.zeros((rows, held), dtype=torch.float64, device=DEV)
    there = dev(((src >= 0) & (src < x_rows)))
    at = dev(np.clip(src, 0, x_rows - 1).astype(np.int64))
    begin = 0
    for k, end in enumerate(ends.tolist()):
        if end > begin:
            picked = q[at[begin:end], :cin].double() * there[begin:end, None]
            z[begin:end] = picked @ codes[k].double().t().contiguous() + bias[k]
        begin = end

    def run(scale, dtype, g):
        s = torch.full((x_rows,), scale, device=DEV)
        y = g.view[:, 1:1 + cout]                      # rows of a wider buffer, an element in
        if e:
            hatq.hatq_experts_int8(lin, q, s, dev(ends), dev(src), y=y)
        else:
            hatq.hatq_linear_int8(lin, q, s, y=y)
        g.check()
        bits = torch.int32 if dtype == torch.float32 else torch.int16
        canary = 0x5A5A5A5A if dtype == torch.float32 else 0x5A5A
        for part in (g.view[:, :1], g.view[:, 1 + cout:]):
            assert bool((part.contiguous().view(bits) == canary).all()), "beside the rows"
        return y

    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        y = run(1.0, dtype, Guarded((rows, cout + 4), dtype))
        if not gated:
            ref = z.float().to(dtype)                  # (float16: infinities past 65504)
            assert torch.equal(y, ref)
            continue
        zs = z * step
        g, u = zs[:, :cout], zs[:, cout:]
        ref = g / (1 + torch.exp(-g)) * u
        rel = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
        floor = {torch.float32: 2.0 ** -120, torch.bfloat16: 2.0 ** -120, torch.float16: 2.0 ** -25}[dtype]
        err = 8 * U * ref.abs()
        assert bool(((y.double() - ref).abs() <= err + rel * (ref.abs() + err) + floor).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cin,cout,e,gated", FORWARDS)
def test_floats(dtype, rows, cin, cout, e, gated):
    rng = np.random.default_rng(rows + cin)
    gen = torch.Generator(device=DEV).manual_seed(cin)
    held, experts = cout * (1 + gated), max(e, 1)
    b = 64 if cin % 64 == 0 else 2
    lin = hatq.hatq_pack_linear(torch.randint(-127, 128, (experts, held, cin), generator=gen, device=DEV).to(torch.int8),
                                torch.rand((experts, held), generator=gen, device=DEV) / 64 / cin ** 0.5,
                                torch.randn((experts, held), generator=gen, device=DEV), hblock=b, gated=bool(gated))
    x_rows = rows // 2 + 1 if e else rows
    wide = torch.randn((x_rows, cin + 5), generator=gen, device=DEV).to(dtype)
    x = wide[:, 3:3 + cin]
    if x_rows > 1:
        x[x_rows - 1, cin // 2] = float("nan")
    g = Guarded((rows, cout), dtype)
    codes = hatq.hatq_token_quant(x, b)
    if e:
        ends, src = dev(ragged(rng, e, rows)), dev(sources(rng, rows, x_rows))
        hatq.hatq_experts_forward(lin, x, ends, src, y=g.view)
        ref = hatq.hatq_experts_int8(lin, *codes, ends, src, out_dtype=dtype)
    else:
        hatq.hatq_linear_forward(lin, x, y=g.view)
        ref = hatq.hatq_linear_int8(lin, *codes, out_dtype=dtype)
    g.check()
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(g.view), nan) and torch.equal(g.view.view(bits)[~nan], ref.view(bits)[~nan])
    if not e and rows > 1:
        assert bool(nan[rows - 1].all()) and not bool(nan[:rows - 1].any())
