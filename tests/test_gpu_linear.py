"""Linear layers over tokens (token codes, the INT8 product, products grouped by expert,
the expert order and the weighted sum) against plain implementations in 64 bits.

Tolerances, derived from the arithmetic (u = 2^-24, the fp32 unit roundoff):
  * codes and scales: bit-exact against the same fp32 butterflies in numpy (IEEE sums,
    products and divisions in a fixed order are the same everywhere).
  * z = fma(float(acc), f, bias), f = fl(s w) / b with b a power of two: f and float(acc)
    are each off by at most u relative, so |z - z64| <= (2u + u^2) |acc f| + u |z|; the
    tests allow 4u |acc f| + 2u |z|.
  * a gated layer: |silu'| < 1.1, so an error d of the gate moves y by at most 1.1 |u_| d
    and one of the value by |silu(g)| d; exp2 of a product rounded to |g| 1.45 u and three
    more operations of at most 2 u each: 2 (|g| + 8) u |y|.
  * the output's rounding: 2^-8 (bfloat16, 8 bits of significand), 2^-11 (float16, or 2^-25 where subnormal).
"""
import numpy as np
import pytest
import torch

from gpu_util import DEV, Guarded, dev, host
from paper_2608_01653_amd import experts, hatq, synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUND = {torch.float32: (U, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


# ---- plain implementations -----------------------------------------------------------

def butterfly(x, b):
    """The order-b Sylvester butterfly of the last axis in x's type, ascending stages."""
    rows = x.shape[0]
    h = 1
    while h < b:
        v = x.reshape(rows, -1, 2, h)
        x = np.stack((v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]), 2).reshape(rows, -1)
        h *= 2
    return x


def token_codes(x, b):
    """(codes int64, scales fp32) of fp32 tokens, the kernel's arithmetic in numpy."""
    with np.errstate(all="ignore"):
        s = butterfly(x.astype(np.float32), b)
        most = np.abs(s).max(axis=1)
        scale = (most / np.float32(127.0)).astype(np.float32)
        scale[scale == 0] = 1.0
        q = np.clip(np.rint(s / scale[:, None]), -127, 127)
        bad = ~np.isfinite(most)
        scale[bad] = np.nan
        q[bad] = 0
    return q.astype(np.int64), scale


def layer64(q, scale, codes, w_scale, bias, b, gated):
    """(y, bound) in 64 bits of rows of codes through one layer, the bound without the
    output's rounding."""
    acc = q @ codes.astype(np.int64).T
    prod = acc * (scale.astype(np.float64)[:, None] * w_scale.astype(np.float64) / b)
    z = prod + bias.astype(np.float64)
    err = 4 * U * np.abs(prod) + 2 * U * np.abs(z)
    if not gated:
        return z, err
    h = z.shape[1] // 2
    g, v, eg, ev = z[:, :h], z[:, h:], err[:, :h], err[:, h:]
    with np.errstate(over="ignore"):
        silu = g / (1 + np.exp(-g))
    y = silu * v
    return y, 1.1 * np.abs(v) * eg + np.abs(silu) * ev + 1.1 * eg * ev + 2 * (np.abs(g) + 8) * U * np.abs(y)


def assert_close(y, ref, err, dtype, what=""):
    rel, floor = ROUND[dtype]
    got = host(y.double())
    assert got.shape == ref.shape
    off = np.abs(got - ref) - (err + rel * (np.abs(ref) + err) + floor)
    ok = bool((off <= 0).all())
    assert ok, f"{what}: {off.max():.3g} past the bound at {np.argwhere(off > 0)[:4].tolist()}"


def make_layer(rng, e, held, cin, bias=True):
    codes = rng.integers(-127, 128, (e, held, cin)).astype(np.int8)
    scale = (rng.uniform(0.5, 1.5, (e, held)) / 64 / np.sqrt(cin)).astype(np.float32)
    b = rng.normal(0, 0.5, (e, held)).astype(np.float32) if bias else np.zeros((e, held), np.float32)
    return codes, scale, b


def pack(layer, b, gated):
    codes, scale, bias = layer
    return hatq.hatq_pack_linear(dev(codes), dev(scale), dev(bias), hblock=b, gated=gated)


def tokens(rng, rows, cin, dtype, pad=0, shift=0):
    """(tensor of `dtype`, its values as fp32): rows in a buffer `pad` wider, `shift` in."""
    x = synth.heavy_tailed_activations(rng, (rows, cin)) if cin > 1 else rng.normal(0, 1, (rows, 1)).astype(np.float32)
    buf = torch.full((rows, cin + pad), 1e4, dtype=dtype, device=DEV)
    t = buf[:, shift:shift + cin]
    t.copy_(dev(np.clip(x, -3e4, 3e4)))
    return t, host(t.float())


# ---- token codes ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cin,b,pad,shift", [
    (1, 1, 1, 0, 0), (3, 7, 1, 2, 1), (5, 62, 2, 0, 0), (4, 68, 4, 1, 1), (9, 1000, 8, 24, 8), (2, 80, 16, 0, 0),
    (7, 96, 32, 8, 0), (1, 320, 64, 0, 0), (66, 192, 64, 3, 3), (130, 128, 128, 0, 0), (1, 4096, 128, 0, 0),
    (3, 4096, 1, 1, 0), (1025, 640, 128, 0, 0), (1030, 1024, 64, 0, 0), (1024, 2048, 128, 8, 8), (1027, 4096, 64, 0, 0),
    (2, 2048, 128, 0, 0), (2, 8192, 128, 0, 0), (1024, 8192, 128, 0, 0), (1, 12288, 64, 0, 0), (1025, 16384, 128, 0, 0),
    (2, 16384, 128, 0, 0), (2, 32768, 128, 0, 0), (2, 65536, 128, 0, 0), (2, 65535, 1, 0, 0)])
def test_token_codes(dtype, rows, cin, b, pad, shift):
    rng = np.random.default_rng(rows * 131 + cin + b)
    x, xf = tokens(rng, rows, cin, dtype, pad, shift)
    ks = (cin + 63) // 64 * 64
    q, s = Guarded((rows, ks), torch.int8), Guarded((rows,), torch.float32)
    hatq.hatq_token_quant(x, b, xq=q.view, scale=s.view)
    q.check("codes")
    s.check("scales")
    ref, scale = token_codes(xf, b)
    assert np.array_equal(host(s.view), scale)
    got = host(q.view).astype(np.int64)
    assert np.array_equal(got[:, :cin], ref)
    assert not got[:, cin:].any()


def test_token_codes_ties_and_ranges():
    """Quotients on and beside half-integers, tiny and huge scales, a zero row."""
    rng = np.random.default_rng(5)
    x = rng.integers(-254, 255, (64, 256)).astype(np.float32) / 2      # halves: ties at scale 1
    x[:, 0] = 127.0
    mult = np.ones((64, 1), np.float32)
    mult[1:40, 0] = 2.0 ** np.linspace(-140, 120, 39).round()
    x = x * mult
    x[50] = 0.0
    x[51] = 0.0
    x[51, 3] = 1e-45     # its scale rounds to 0
    x[52] = np.nextafter(x[52], np.float32(np.inf))
    x[53] = np.nextafter(x[53], np.float32(-np.inf))
    for b in (1, 8):
        q, s = hatq.hatq_token_quant(dev(x), b)
        ref, scale = token_codes(x, b)
        assert np.array_equal(host(s), scale, equal_nan=True)     # (a sum of eight of the largest overflows)
        assert np.array_equal(host(q).astype(np.int64), ref)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cin", [256, 4096, 16384])
def test_token_not_finite(dtype, cin):
    """A token with a NaN or an infinity has a NaN scale and codes 0; the others theirs."""
    rng = np.random.default_rng(cin)
    x, xf = tokens(rng, 9, cin, dtype)
    for row, v in ((1, np.nan), (3, np.inf), (4, -np.inf)):
        x[row, int(rng.integers(cin))] = v
    q, s = hatq.hatq_token_quant(x, 64)
    ref, scale = token_codes(host(x.float()), 64)
    assert np.array_equal(np.isnan(scale), np.isin(np.arange(9), (1, 3, 4)))
    assert np.array_equal(host(s), scale, equal_nan=True)
    assert np.array_equal(host(q).astype(np.int64), ref)
    if dtype is torch.float32:   # finite, but the transform overflows
        x = torch.full((1, 256), 3e38, device=DEV)
        q, s = hatq.hatq_token_quant(x, 4)
        assert np.isnan(host(s)).all() and not host(q).any()


# ---- weights --------------------------------------------------------------------------------

def unpack(lin):
    """(codes [e][held][cin], scales, bias) of prepared weights, from the layout's definition."""
    w, e = lin.w, lin.experts
    n = e * w.cout_pad * w.k_stride
    blocks = host(lin.buf[:n]).reshape(e, w.cout_pad // 16, w.k_stride // 64, 4, 16, 16)
    cols = blocks.transpose(0, 1, 4, 2, 3, 5).reshape(e, w.cout_pad, w.k_stride)

    def floats(ptr):
        off = ptr - lin.buf.data_ptr()
        return host(lin.buf[off:off + 4 * e * w.cout_pad].view(torch.float32)).reshape(e, w.cout_pad)
    scale, bias = floats(w.w_scale), floats(w.bias)
    if w.gated:
        p = np.concatenate([(np.arange(lin.cout) // 32) * 64 + np.arange(lin.cout) % 32 + 32 * v for v in (0, 1)])
    else:
        p = np.arange(lin.cout)
    rest = np.setdiff1d(np.arange(w.cout_pad), p)
    assert not cols[:, rest].any() and not scale[:, rest].any() and not bias[:, rest].any()
    assert not cols[:, :, lin.cin:].any()
    return cols[:, p, :lin.cin], scale[:, p], bias[:, p]


@pytest.mark.parametrize("e,held,cin,gated", [(1, 1, 1, False), (1, 33, 70, False), (3, 48, 64, True),
                                              (2, 66, 129, True), (1, 2, 5, True), (4, 100, 256, False)])
def test_pack(e, held, cin, gated):
    rng = np.random.default_rng(held)
    layer = make_layer(rng, e, held, cin)
    got = unpack(pack(layer, 1, gated))
    for a, r in zip(got, layer):
        assert np.array_equal(a, r)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("e,held,cin,b,gated", [(1, 40, 128, 64, False), (2, 34, 96, 32, True), (1, 5, 33, 1, False),
                                                (1, 16, 256, 128, False)])
def test_prepare(orc, dtype, e, held, cin, b, gated):
    """Codes, scales and bias of float weights, as the oracle prepares a 1x1 layer's."""
    rng = np.random.default_rng(cin)
    w = torch.from_numpy(synth.student_t_weights(rng, (e, held, cin)))
    w[0, held // 2] = 0.0
    w = w.to(dtype).to(DEV)
    bias = rng.normal(0, 1, (e, held)).astype(np.float32)
    codes, scale, got_bias = unpack(hatq.hatq_prepare_linear(w, dev(bias), hblock=b, gated=gated))
    wf = host(w.float())
    for i in range(e):
        ref = orc.prepare_weights(np.ascontiguousarray(wf[i].reshape(held, cin, 1, 1)), bias[i], cin=cin, cout=held,
                                  k=1, stride=1, pad=0, form="DH", hblock=b)
        assert np.array_equal(scale[i], ref.w_scale[:held])
        assert np.array_equal(codes[i], ref.wq.reshape(held, -1)[:, :cin])
    assert np.array_equal(got_bias, bias)


# ---- the product ---------------------------------------------------------------------------

SHAPES = [  # rows, cin, cout
    (1, 1, 1), (1, 64, 16), (1, 320, 192), (2, 65, 17), (15, 200, 33), (16, 1024, 48), (17, 513, 100), (31, 64, 1),
    (33, 4160, 40), (64, 700, 130), (65, 128, 65), (77, 1000, 1001), (128, 64, 128), (129, 127, 257), (200, 2048, 31),
    (255, 192, 320), (300, 576, 260), (513, 320, 129), (1100, 448, 700)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_product(rows, cin, cout, gated):
    """Random codes, fp32 outputs with guard bytes around them."""
    rng = np.random.default_rng(rows + 7 * cin + cout)
    held = 2 * cout if gated else cout
    layer = make_layer(rng, 1, held, cin)
    lin = pack(layer, 1, gated)
    ks = lin.k_stride
    q = rng.integers(-127, 128, (rows, ks)).astype(np.int8)     # bytes past cin meet zero weights
    s = rng.uniform(0.001, 0.01, rows).astype(np.float32)
    y = Guarded((rows, cout), torch.float32)
    hatq.hatq_linear_int8(lin, dev(q), dev(s), y=y.view)
    y.check()
    ref, err = layer64(q[:, :cin].astype(np.int64), s, *(a[0] for a in layer), 1, gated)
    assert_close(y.view, ref, err, torch.float32)


# Large shapes at the tiles' edges (not every kernel: test_gpu_linear_paths.py has those): the
# sums stay below 2^24, so that with scales of 1 and no bias float32 outputs are the integers
# themselves.
LARGE = [(20, 8192, 100), (45, 2048, 4100), (65, 4096, 1030), (129, 16384, 200), (190, 4096, 4097), (385, 4032, 2050), (515, 4096, 4096),
         (1025, 4096, 2100), (1000, 1000, 6000), (2050, 4096, 4100), (4097, 1088, 4100), (9000, 320, 700), (6145, 2048, 1300),
         (70001, 64, 40)]


def exact_sums(q, codes):
    """q codes^T on the device, exact: integers below 2^53 in float64."""
    return q.double() @ codes.double().t().contiguous()


@pytest.mark.parametrize("rows,cin,cout", LARGE)
def test_product_large(rows, cin, cout):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    lim = max(1, int((2 ** 24 / cin) ** 0.5) - 1)
    codes = torch.randint(-lim, lim + 1, (cout, cin), generator=gen, device=DEV).to(torch.int8)
    lin = hatq.hatq_pack_linear(codes, torch.ones(cout, device=DEV))
    q = torch.zeros((rows, lin.k_stride), dtype=torch.int8, device=DEV)
    q[:, :cin] = torch.randint(-lim, lim + 1, (rows, cin), generator=gen, device=DEV)
    y = Guarded((rows, cout), torch.float32)
    hatq.hatq_linear_int8(lin, q, torch.ones(rows, device=DEV), y=y.view)
    y.check()
    ref = exact_sums(q[:, :cin], codes)
    assert torch.equal(y.view.double(), ref)
    # one scale, halves and bfloat16 the same values rounded once; a gated layer its unit
    for dtype in (torch.float16, torch.bfloat16):
        got = hatq.hatq_linear_int8(lin, q, torch.full((rows,), 2.0 ** -12, device=DEV), out_dtype=dtype)
        assert torch.equal(got, (ref * 2.0 ** -12).float().to(dtype))


@pytest.mark.parametrize("rows,cin,cout", [(45, 2048, 2050), (190, 4096, 2049), (385, 4032, 1030), (1025, 4096, 1050), (2050, 4096, 2050),
                                           (4097, 1088, 2050)])
def test_product_large_gated(rows, cin, cout):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    lim = max(1, int((2 ** 24 / cin) ** 0.5) - 1)
    codes = torch.randint(-lim, lim + 1, (2 * cout, cin), generator=gen, device=DEV).to(torch.int8)
    lin = hatq.hatq_pack_linear(codes, torch.full((2 * cout,), 2.0 ** -10, device=DEV), gated=True)
    q = torch.zeros((rows, lin.k_stride), dtype=torch.int8, device=DEV)
    q[:, :cin] = torch.randint(-lim, lim + 1, (rows, cin), generator=gen, device=DEV)
    y = hatq.hatq_linear_int8(lin, q, torch.full((rows,), 2.0 ** -8, device=DEV))
    z = exact_sums(q[:, :cin], codes) * 2.0 ** -18          # exact in float32 too
    g, u = z[:, :cout], z[:, cout:]
    ref = g * torch.sigmoid(g) * u
    assert bool(((y.double() - ref).abs() <= 2 * (g.abs() + 8) * U * ref.abs() + 2.0 ** -120).all())


@pytest.mark.parametrize("e,rows,cin,cout", [(3, 900, 2048, 1030), (40, 3000, 1088, 600), (8, 9001, 2048, 1100), (100, 20000, 576, 520),
                                             (2, 5000, 4096, 2050), (64, 64, 4096, 130), (16, 700, 2048, 2050), (300, 40000, 128, 100)])
def test_grouped_large(e, rows, cin, cout):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    rng = np.random.default_rng(rows)
    lim = max(1, int((2 ** 24 / cin) ** 0.5) - 1)
    codes = torch.randint(-lim, lim + 1, (e, cout, cin), generator=gen, device=DEV).to(torch.int8)
    lin = hatq.hatq_pack_linear(codes, torch.ones((e, cout), device=DEV))
    x_rows = rows // 2 + 1
    q = torch.zeros((x_rows, lin.k_stride), dtype=torch.int8, device=DEV)
    q[:, :cin] = torch.randint(-lim, lim + 1, (x_rows, cin), generator=gen, device=DEV)
    ends = np.cumsum(rng.multinomial(rows - 7, rng.dirichlet(np.full(e, 0.5))))      # seven rows left over
    src = torch.randint(0, x_rows, (rows,), generator=gen, device=DEV).to(torch.int32)
    y = Guarded((rows, cout), torch.float32)
    hatq.hatq_experts_int8(lin, q, torch.ones(x_rows, device=DEV), dev(ends.astype(np.int32)), src, y=y.view)
    y.check()
    begin = 0
    for k, end in enumerate(ends.tolist()):
        if end > begin:
            assert torch.equal(y.view[begin:end].double(), exact_sums(q[src[begin:end].long(), :cin], codes[k])), k
        begin = end
    assert not bool(y.view[begin:].any())


@pytest.mark.parametrize("rows,cout", [(3, 50), (40, 66), (150, 130), (300, 512)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 0), (8, 8), (5, 3)])
def test_product_output_rows(rows, cout, dtype, pad, shift):
    """Every type, into rows of a wider buffer at any alignment; nothing beside them is
    written."""
    rng = np.random.default_rng(rows + cout)
    cin = 192
    layer = make_layer(rng, 1, cout, cin)
    lin = pack(layer, 64, False)
    q = rng.integers(-127, 128, (rows, cin)).astype(np.int8)
    s = rng.uniform(0.001, 0.01, rows).astype(np.float32)
    g = Guarded((rows, cout + pad), dtype)
    before = g.view.clone()
    y = g.view[:, shift:shift + cout]
    hatq.hatq_linear_int8(lin, dev(q), dev(s), y=y)
    g.check()
    bits = torch.int32 if dtype == torch.float32 else torch.int16      # (the canary is a NaN in some types)
    for part in (slice(0, shift), slice(shift + cout, None)):
        assert torch.equal(g.view[:, part].view(bits), before[:, part].view(bits))
    ref, err = layer64(q.astype(np.int64), s, *(a[0] for a in layer), 64, False)
    assert_close(y, ref, err, dtype)


@pytest.mark.parametrize("rows,cin,cout", [(1, 65536, 16), (70, 65536, 24)])
def test_product_longest_contraction(rows, cin, cout):
    """Codes of 127 everywhere: the largest sum, 65536 * 127^2, in INT32."""
    codes = np.full((1, cout, cin), 127, np.int8)
    codes[0, 1::2] = -127
    layer = (codes, np.full((1, cout), 1e-4, np.float32), np.zeros((1, cout), np.float32))
    lin = pack(layer, 1, False)
    q = np.full((rows, cin), 127, np.int8)
    s = np.full(rows, 0.5, np.float32)
    y = hatq.hatq_linear_int8(lin, dev(q), dev(s))
    ref, err = layer64(q.astype(np.int64), s, *(a[0] for a in layer), 1, False)
    assert_close(y, ref, err, torch.float32)


def test_product_nan_scale_stays_in_its_row():
    rng = np.random.default_rng(3)
    for rows in (5, 40, 200, 600):
        layer = make_layer(rng, 1, 96, 128)
        lin = pack(layer, 1, False)
        q = rng.integers(-127, 128, (rows, 128)).astype(np.int8)
        s = rng.uniform(0.001, 0.01, rows).astype(np.float32)
        s[rows // 2] = np.nan
        y = host(hatq.hatq_linear_int8(lin, dev(q), dev(s)))
        nan = np.isnan(y)
        assert nan[rows // 2].all() and not np.delete(nan, rows // 2, 0).any()


@pytest.mark.parametrize("rows,cin,cout,b,gated,dtype", [
    (1, 320, 192, 64, False, torch.bfloat16), (1, 4096, 512, 128, False, torch.bfloat16),
    (13, 1024, 300, 128, True, torch.float16), (77, 1000, 101, 8, False, torch.float32),
    (600, 320, 320, 64, False, torch.float32), (1500, 256, 520, 64, True, torch.bfloat16),
    (3, 130, 70, 2, True, torch.float32), (260, 100, 60, 1, True, torch.float16)])
def test_forward(rows, cin, cout, b, gated, dtype):
    rng = np.random.default_rng(rows)
    layer = make_layer(rng, 1, 2 * cout if gated else cout, cin)
    lin = pack(layer, b, gated)
    x, xf = tokens(rng, rows, cin, dtype, 8, 8)
    y = hatq.hatq_linear_forward(lin, x)
    assert y.dtype == dtype
    q, s = token_codes(xf, b)
    ref, err = layer64(q, s, *(a[0] for a in layer), b, gated)
    assert_close(y, ref, err, dtype)
    wide = hatq.hatq_linear_forward(lin, x, out_dtype=torch.float32)
    assert_close(wide, ref, err, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cin,cout,b,pad", [
    (1, 1, 1, 1, 0), (1, 64, 16, 64, 0), (2, 500, 40, 4, 1), (16, 512, 33, 128, 0), (9, 640, 20, 128, 8), (16, 1024, 50, 64, 0),
    (1, 1024, 70, 64, 0), (3, 1100, 17, 2, 3), (4, 4096, 64, 128, 0), (3, 4097, 24, 1, 0), (2, 8192, 16, 128, 0), (1, 16384, 40, 128, 0),
    (1, 16000, 16, 64, 8), (1, 20000, 16, 32, 0), (17, 256, 30, 64, 0), (300, 320, 200, 64, 0), (9001, 192, 70, 64, 0),
    (8300, 1000, 24, 8, 1), (33, 1024, 1500, 128, 0), (20, 2048, 200, 128, 0), (100, 1900, 70, 4, 3), (9, 2048, 40, 64, 0)])
def test_forward_is_its_two_steps(dtype, gated, rows, cin, cout, b, pad):
    """Floats in and codes in give the same bits, whichever kernels a call takes."""
    rng = np.random.default_rng(cin + rows)
    lin = pack(make_layer(rng, 1, 2 * cout if gated else cout, cin), b, gated)
    x, _ = tokens(rng, rows, cin, dtype, pad, pad // 2)
    if rows > 1:
        x[rows - 1, cin // 2] = float("inf")
    g = Guarded((rows, cout), dtype)
    hatq.hatq_linear_forward(lin, x, y=g.view)
    g.check()
    ref = hatq.hatq_linear_int8(lin, *hatq.hatq_token_quant(x, b), out_dtype=dtype)
    assert torch.equal(g.view.nan_to_num(nan=7.0), ref.nan_to_num(nan=7.0))
    assert rows == 1 or bool(torch.isnan(ref[rows - 1]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("e,rows,cin,cout,gated", [(64, 48, 2048, 40, False), (32, 96, 512, 48, True), (8, 20, 256, 17, False), (4, 64, 960, 64, True),
                                                   (200, 3, 4096, 16, False), (16, 300, 128, 16, False)])
@pytest.mark.parametrize("skew", [False, True])
def test_grouped_forward_is_its_two_steps(dtype, e, rows, cin, cout, gated, skew):
    rng = np.random.default_rng(cin + rows)
    lin = pack(make_layer(rng, e, 2 * cout if gated else cout, cin), 64, gated)
    x, _ = tokens(rng, rows // 2 + 1, cin, dtype)
    ends = np.cumsum(rng.multinomial(rows - rows // 8, rng.dirichlet(np.full(e, 0.05 if skew else 5.0)))).astype(np.int32)
    src = rng.integers(-1, x.shape[0] + 1, rows).astype(np.int32)
    g = Guarded((rows, cout), dtype)
    hatq.hatq_experts_forward(lin, x, dev(ends), dev(src), y=g.view)
    g.check()
    ref = hatq.hatq_experts_int8(lin, *hatq.hatq_token_quant(x, 64), dev(ends), dev(src), out_dtype=dtype)
    assert torch.equal(g.view, ref)


# ---- grouped by expert ----------------------------------------------------------------------

def grouped64(q, s, layer, ends, src, rows, b, gated):
    """Row by row from the definition, any ends and src."""
    codes, scale, bias = layer
    e_of = np.full(rows, -1)
    begin = 0
    for e, end in enumerate(ends):
        end = max(begin, min(int(end), rows))
        e_of[begin:end] = e
        begin = end
    ref = np.zeros((rows, codes.shape[1] // (2 if gated else 1)))
    err = np.zeros_like(ref)
    for e in range(codes.shape[0]):
        at = np.nonzero(e_of == e)[0]
        if not at.size:
            continue
        t = at if src is None else src[at]
        empty = (t < 0) | (t >= q.shape[0])
        t = np.where(empty, 0, t)
        qe, se = np.where(empty[:, None], 0, q[t]), np.where(empty, 1.0, s[t])
        ref[at], err[at] = layer64(qe, se.astype(np.float32), codes[e], scale[e], bias[e], b, gated)
    return ref, err


GROUPS = {
    "even": lambda rng, e, rows: np.arange(1, e + 1) * rows // e,
    "one expert": lambda rng, e, rows: np.where(np.arange(e) >= e // 2, rows, 0),
    "ragged": lambda rng, e, rows: np.cumsum(rng.multinomial(rows, rng.dirichlet(np.full(e, 0.3)))),
    "rows left over": lambda rng, e, rows: np.cumsum(rng.multinomial(rows // 2, np.full(e, 1 / e))),
    "none": lambda rng, e, rows: np.zeros(e),
    "past the rows": lambda rng, e, rows: np.arange(1, e + 1) * rows,
    "unordered, negative": lambda rng, e, rows: rng.integers(-rows, 2 * rows, e),
}


@pytest.mark.parametrize("ends", list(GROUPS))
@pytest.mark.parametrize("e,rows,cin,cout,gated", [(1, 5, 64, 40, False), (7, 40, 192, 66, True), (64, 48, 128, 40, False),
                                                   (100, 33, 64, 20, True), (3, 500, 320, 130, False),
                                                   (5, 1500, 128, 300, True), (1024, 700, 64, 16, False)])
def test_grouped(ends, e, rows, cin, cout, gated):
    rng = np.random.default_rng(e + rows)
    layer = make_layer(rng, e, 2 * cout if gated else cout, cin)
    lin = pack(layer, 1, gated)
    ends = GROUPS[ends](rng, e, rows).astype(np.int32)
    x_rows = rows // 3 + 1
    q = rng.integers(-127, 128, (x_rows, cin)).astype(np.int8)
    s = rng.uniform(0.001, 0.01, x_rows).astype(np.float32)
    src = rng.integers(0, x_rows, rows).astype(np.int32)
    if rows > 4:
        src[rng.integers(0, rows, 3)] = (-1, x_rows, 2 ** 31 - 1)
    y = Guarded((rows, cout), torch.float32)
    hatq.hatq_experts_int8(lin, dev(q), dev(s), dev(ends), dev(src), y=y.view)
    y.check()
    ref, err = grouped64(q.astype(np.int64), s, layer, ends, src, rows, 1, gated)
    assert_close(y.view, ref, err, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,e", [(9, 4), (300, 4), (2100, 3)])
def test_grouped_forward(dtype, rows, e):
    """Floats in, in place rows (no src)."""
    rng = np.random.default_rng(rows)
    cin, cout, b = 256, 200, 128
    layer = make_layer(rng, e, cout, cin)
    lin = pack(layer, b, False)
    x, xf = tokens(rng, rows, cin, dtype)
    ends = GROUPS["ragged"](rng, e, rows).astype(np.int32)
    y = hatq.hatq_experts_forward(lin, x, dev(ends))
    q, s = token_codes(xf, b)
    ref, err = grouped64(q, s, layer, ends, None, rows, b, False)
    assert_close(y, ref, err, dtype)


# ---- order and sum ------------------------------------------------------------------------------

def order_ref(ids, e):
    flat = ids.reshape(-1).astype(np.int64)
    ok = (flat >= 0) & (flat < e)
    at = np.nonzero(ok)[0]
    at = at[np.argsort(flat[at], kind="stable")]
    src = np.full(flat.size, -1)
    src[:at.size] = at // ids.shape[1]
    pos = np.full(flat.size, -1)
    pos[at] = np.arange(at.size)
    return np.cumsum(np.bincount(flat[ok], minlength=e)), src, pos.reshape(ids.shape)


@pytest.mark.parametrize("tokens_,topk,e", [(1, 1, 1), (1, 4, 64), (24, 4, 32), (63, 1, 3), (64, 1, 1024), (700, 3, 5),
                                            (1024, 1, 7), (1025, 1, 7), (5000, 6, 200), (3, 2, 1024), (100001, 3, 17),
                                            (0, 2, 4)])
@pytest.mark.parametrize("masked", [False, True])
def test_order(tokens_, topk, e, masked):
    rng = np.random.default_rng(tokens_ + e)
    ids = rng.integers(-2 if masked else 0, e + 2 if masked else e, (tokens_, topk)).astype(np.int32)
    if masked and tokens_:
        ids[0, 0], ids[-1, -1] = -2 ** 31, 2 ** 31 - 1
    g = [Guarded((n,), torch.int32) for n in (e, tokens_ * topk, tokens_ * topk)]
    hatq.hatq_expert_order(dev(ids).view(tokens_, topk), e, ends=g[0].view, src=g[1].view, pos=g[2].view)
    for t, r in zip(g, order_ref(ids, e)):
        t.check()
        assert np.array_equal(host(t.view), r.reshape(-1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens_,topk,cols,pad", [(1, 1, 1, 0), (7, 3, 130, 0), (50, 4, 64, 1), (9, 2, 513, 3), (300, 6, 256, 4)])
def test_combine(dtype, tokens_, topk, cols, pad):
    rng = np.random.default_rng(cols)
    rows = tokens_ * topk
    h = rng.normal(0, 1, (rows, cols + pad)).astype(np.float32)
    pos = rng.permutation(rows).reshape(tokens_, topk).astype(np.int32)
    w = rng.uniform(0, 1, (tokens_, topk)).astype(np.float32)
    if topk > 1:
        pos[0] = -1                       # a token with no row
        pos[-1, 1] = rows                 # and a row that is not there
    y = Guarded((tokens_, cols), dtype)
    hatq.hatq_expert_combine(dev(h)[:, :cols], dev(pos), dev(w), y=y.view)
    y.check()
    ok = (pos >= 0) & (pos < rows)
    terms = np.where(ok, w, 0.0).astype(np.float64)[:, :, None] * h[np.where(ok, pos, 0), :cols]
    # topk fused multiply-adds of fp32: each rounds a partial sum
    assert_close(y.view, terms.sum(1), topk * U * np.abs(terms).sum(1), dtype)


# ---- together ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens_,topk,e,width,hidden,b", [(1, 2, 4, 128, 64, 64), (24, 4, 32, 256, 128, 64), (200, 3, 5, 192, 320, 64),
                                                           (900, 2, 3, 128, 256, 128)])
def test_expert_block(tokens_, topk, e, width, hidden, b):
    """Each step of the block against its definition on the step before's own output (a
    last bit of the hidden rows may move a code, so the whole is compared by steps)."""
    rng = np.random.default_rng(width)
    l_in, l_out = make_layer(rng, e, 2 * hidden, width), make_layer(rng, e, width, hidden)
    p_in, p_out = pack(l_in, b, True), pack(l_out, b, False)
    x, xf = tokens(rng, tokens_, width, torch.bfloat16)
    ids = np.stack([rng.permutation(e)[:topk] for _ in range(tokens_)]).astype(np.int32)
    w = rng.dirichlet(np.ones(topk), tokens_).astype(np.float32)
    y = experts.ExpertMLP(p_in, p_out)(x, dev(ids), dev(w))
    assert y.dtype == torch.bfloat16
    ends, src, pos = order_ref(ids, e)
    hid = hatq.hatq_experts_forward(p_in, x, dev(ends.astype(np.int32)), dev(src.astype(np.int32)), out_dtype=torch.float32)
    ref, err = grouped64(*token_codes(xf, b), l_in, ends, src, tokens_ * topk, b, True)
    assert_close(hid, ref, err, torch.float32)
    ref, err = grouped64(*token_codes(host(hid), b), l_out, ends, None, tokens_ * topk, b, False)
    wt = w.astype(np.float64)[:, :, None]
    total, bound = (ref[pos] * wt).sum(1), (err[pos] * wt).sum(1) + topk * U * (np.abs(ref[pos]) * wt).sum(1)
    assert_close(y, total, bound, torch.bfloat16)


def test_masked_pairs_add_nothing():
    rng = np.random.default_rng(8)
    p_in, p_out = pack(make_layer(rng, 4, 128, 64), 1, True), pack(make_layer(rng, 4, 64, 64), 1, False)
    mlp = experts.ExpertMLP(p_in, p_out)
    x, _ = tokens(rng, 30, 64, torch.float32)
    ids = rng.integers(0, 4, (30, 3)).astype(np.int32)
    w = rng.uniform(0, 1, (30, 3)).astype(np.float32)
    masked = ids.copy()
    masked[:, 2] = -1
    w0 = w.copy()
    w0[:, 2] = 0
    assert torch.equal(mlp(x, dev(masked), dev(w)), mlp(x, dev(ids), dev(w0)))
    assert not host(mlp(x, dev(np.full_like(ids, -1)), dev(w))).any()


# ---- streams, graphs, refusals --------------------------------------------------------------------

def test_other_stream_and_graph():
    """The same results on another stream and from a captured graph, replayed with other
    inputs in the same buffers."""
    rng = np.random.default_rng(9)
    layer = make_layer(rng, 3, 160, 128)
    lin = pack(layer, 64, False)
    x, _ = tokens(rng, 50, 128, torch.bfloat16)
    ends = dev(np.array([10, 10, 45], np.int32))
    ref = hatq.hatq_experts_forward(lin, x, ends)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hatq.hatq_experts_forward(lin, x, ends, stream=side)
    side.synchronize()
    assert torch.equal(got, ref)
    y = torch.empty_like(ref)
    ws = torch.empty(hatq.hatq_linear_ws_bytes(lin, 50), dtype=torch.int8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hatq.hatq_experts_forward(lin, x, ends, y=y, ws=ws)
    for k in range(4):
        x.copy_(tokens(rng, 50, 128, torch.bfloat16)[0])
        ends.copy_(dev(np.array([5 * k, 20, 50 - k], np.int32)))
        ref = hatq.hatq_experts_forward(lin, x, ends)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref), k


def test_no_rows():
    rng = np.random.default_rng(1)
    lin = pack(make_layer(rng, 1, 16, 64), 1, False)
    x = torch.empty((0, 64), device=DEV)
    assert hatq.hatq_linear_forward(lin, x).shape == (0, 16)
    assert hatq.hatq_token_quant(x)[0].shape == (0, 64)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    assert hatq.hatq_experts_forward(lin, torch.ones((2, 64), device=DEV), dev(np.zeros(1, np.int32)), none).shape == (0, 16)
    y = hatq.hatq_expert_combine(torch.empty((0, 8), device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV),
                                 torch.ones((3, 2), device=DEV))
    assert y.shape == (3, 8) and not host(y).any()


def test_refusals():
    rng = np.random.default_rng(1)
    lin = pack(make_layer(rng, 1, 16, 64), 1, False)
    two = pack(make_layer(rng, 2, 16, 64), 1, False)
    x = torch.zeros((4, 64), device=DEV)
    ends = dev(np.array([4], np.int32))
    bad = [
        lambda: hatq.hatq_linear_forward(lin, x[:, :63]),                       # other width
        lambda: hatq.hatq_linear_forward(lin, torch.zeros((64, 4), device=DEV).t()),   # elements not adjacent
        lambda: hatq.hatq_linear_forward(lin, x[:1].expand(4, 64)),             # rows that overlap
        lambda: hatq.hatq_linear_forward(lin, x.double()),
        lambda: hatq.hatq_linear_forward(lin, x.cpu()),
        lambda: hatq.hatq_linear_forward(lin, x, y=torch.empty((3, 16), device=DEV)),
        lambda: hatq.hatq_linear_forward(lin, x, y=torch.empty((4, 17), device=DEV)),
        lambda: hatq.hatq_linear_int8(lin, torch.zeros((4, 128), dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV)),
        lambda: hatq.hatq_linear_int8(lin, torch.zeros((4, 64), dtype=torch.int8, device=DEV), torch.zeros(3, device=DEV)),
        lambda: hatq.hatq_experts_forward(two, x, ends),                        # an end for each expert
        lambda: hatq.hatq_experts_forward(lin, x, ends.long()),
        lambda: hatq.hatq_experts_forward(lin, x, ends, ends.view(1, 1)),
        lambda: hatq.hatq_pack_linear(torch.zeros((3, 8), dtype=torch.int8, device=DEV), torch.ones(3, device=DEV), gated=True),
        lambda: hatq.hatq_expert_order(torch.zeros((2, 2), device=DEV), 4),
        lambda: hatq.hatq_expert_combine(x.half(), torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.ones((1, 1), device=DEV)),
        lambda: experts.ExpertMLP(lin, lin),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    refused = [
        (lambda: hatq.hatq_linear_forward(two, x), hatq.HATQ_EINVAL),           # experts need ends
        (lambda: hatq.hatq_token_quant(x, 3), hatq.HATQ_EINVAL),
        (lambda: hatq.hatq_token_quant(x, 192), hatq.HATQ_EUNSUPPORTED),
        (lambda: hatq.hatq_token_quant(x, 128), hatq.HATQ_EUNSUPPORTED),        # 64 % 128
        (lambda: hatq.hatq_linear_forward(lin, torch.zeros((17, 64), device=DEV), ws=torch.empty(256, dtype=torch.int8, device=DEV)),
         hatq.HATQ_EWORKSPACE),
        (lambda: hatq.hatq_experts_forward(lin, x, ends, ws=torch.empty(256, dtype=torch.int8, device=DEV)), hatq.HATQ_EWORKSPACE),
        (lambda: hatq.hatq_expert_order(torch.zeros((2, 2), dtype=torch.int32, device=DEV), 1025), hatq.HATQ_EUNSUPPORTED),
        (lambda: hatq.hatq_pack_linear(torch.zeros((4, 8), dtype=torch.int8, device=DEV), torch.ones(4, device=DEV), hblock=16),
         hatq.HATQ_EUNSUPPORTED),
    ]
    for f, status in refused:
        with pytest.raises(hatq.HatqError) as e:
            f()
        assert e.value.status == status


# Few tiles and a long contraction: rows in tiles of 32, the contraction split in the block
# with steps left over, one step for some groups of waves, none for others.
DEEP = [(200, 4096, 1030), (513, 2560, 640), (965, 6656, 330), (33, 8192, 2049), (410, 4160, 513), (225, 12000, 65), (1030, 2600, 97),
        (300, 192, 300), (270, 128, 600), (259, 64, 700)]


@pytest.mark.parametrize("rows,cin,cout", DEEP)
def test_product_deep(rows, cin, cout):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    lim = max(1, int((2 ** 24 / cin) ** 0.5) - 1)
    codes = torch.randint(-lim, lim + 1, (cout, cin), generator=gen, device=DEV).to(torch.int8)
    lin = hatq.hatq_pack_linear(codes, torch.ones(cout, device=DEV))
    q = torch.zeros((rows, lin.k_stride), dtype=torch.int8, device=DEV)
    q[:, :cin] = torch.randint(-lim, lim + 1, (rows, cin), generator=gen, device=DEV)
    y = Guarded((rows, cout), torch.float32)
    hatq.hatq_linear_int8(lin, q, torch.ones(rows, device=DEV), y=y.view)
    y.check()
    assert torch.equal(y.view.double(), exact_sums(q[:, :cin], codes))


@pytest.mark.parametrize("rows,cin,cout", [(500, 2560, 320), (965, 6656, 161), (40, 8192, 1030), (300, 320, 300)])
def test_product_deep_gated(rows, cin, cout):
    test_product_large_gated(rows, cin, cout)


@pytest.mark.parametrize("e,rows,cin,cout", [(2, 400, 4096, 500), (4, 47, 8192, 47), (12, 67, 7710, 31), (57, 89, 8192, 45), (7, 330, 6000, 130),
                                             (25, 65, 4160, 70), (3, 240, 2560, 700)])
def test_grouped_deep(e, rows, cin, cout):
    test_grouped_large(e, rows, cin, cout)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cin,cout,e", [
    (1, 700, 33, 1), (5, 2560, 70, 1), (40, 4096, 130, 1), (300, 192, 90, 1), (500, 4096, 514, 1), (700, 2100, 1029, 1), (2100, 2304, 1030, 1),
    (4100, 2304, 2054, 1), (30, 130, 21, 4), (90, 4096, 70, 6), (700, 2304, 130, 3), (3000, 2304, 300, 2)])
def test_any_address(dtype, rows, cin, cout, e):
    """Rows in and out at every offset of an element and odd strides give the same bits."""
    rng = np.random.default_rng(cin + rows)
    layer = make_layer(rng, e, cout, cin)
    lin = pack(layer, 1, False)
    x = torch.randn((rows, cin), generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV).to(dtype)
    if e > 1:
        ends = dev(np.sort(rng.integers(0, rows + 1, e)).astype(np.int32))
        src = dev(rng.integers(0, rows, rows).astype(np.int32))

        def run(x, y):
            return hatq.hatq_experts_forward(lin, x, ends, src, y=y)
    else:
        def run(x, y):
            return hatq.hatq_linear_forward(lin, x, y=y)
    want = run(x, torch.empty((rows, cout), dtype=dtype, device=DEV))
    for offset, wider in ((1, 1), (3, 5), (2, 2), (5, 7)):
        xs = torch.zeros(offset + rows * (cin + wider), dtype=dtype, device=DEV)
        xv = xs.as_strided((rows, cin), (cin + wider, 1), offset)
        xv.copy_(x)
        ys = torch.full((offset + rows * (cout + wider) + 16,), 7.0, dtype=dtype, device=DEV)
        yv = ys.as_strided((rows, cout), (cout + wider, 1), offset)
        run(xv, yv)
        assert torch.equal(yv, want)
        yv.fill_(7.0)
        assert bool((ys == 7.0).all())           # nothing beside the rows was written


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols", [1, 3, 4, 7, 130])
def test_combine_any_address(dtype, cols):
    rng = np.random.default_rng(cols)
    h = torch.randn((60, cols), generator=torch.Generator(device=DEV).manual_seed(cols), device=DEV)
    pos = dev(rng.integers(0, 60, (25, 3)).astype(np.int32))
    weights = torch.rand((25, 3), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    want = hatq.hatq_expert_combine(h, pos, weights, out_dtype=dtype)
    for offset, wider in ((1, 1), (3, 2)):
        hv = torch.zeros(offset + 60 * (cols + wider), device=DEV).as_strided((60, cols), (cols + wider, 1), offset)
        hv.copy_(h)
        ys = torch.full((offset + 25 * (cols + wider) + 8,), 7.0, dtype=dtype, device=DEV)
        yv = ys.as_strided((25, cols), (cols + wider, 1), offset)
        hatq.hatq_expert_combine(hv, pos, weights, y=yv)
        assert torch.equal(yv, want)
        yv.fill_(7.0)
        assert bool((ys == 7.0).all())
