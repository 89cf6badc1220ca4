"""Plain implementations in numpy of the 4-bit cache and the attention over it."""
import numpy as np
import torch

from gpu_util import DEV, dev
from paper_2608_01653_amd import hatq

U = 2.0 ** -24
# half a step relative to the value, and below the type's normal numbers, which start at
# 2^-126 for both of the first, in itself (float32 may be taken as 0 there)
ROUND = {torch.float32: (U, 2.0 ** -126), torch.bfloat16: (2.0 ** -8, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def butterfly(x, b):
    """The order-b Sylvester butterfly of the last axis in x's type, ascending stages."""
    shape, h = x.shape, 1
    while h < b:
        v = x.reshape(-1, 2, h)
        x = np.stack((v[:, 0] + v[:, 1], v[:, 0] - v[:, 1]), 1)
        h *= 2
    return x.reshape(shape)


def to_bf16(x):
    """float32 rounded half to even to bfloat16, as float32."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def quantize(x, b):
    """(codes, scale of each channel) of heads [..., dim] of float32, the kernel's arithmetic."""
    with np.errstate(all="ignore"):
        s = butterfly(x.astype(np.float32), b)
        scale = np.empty_like(s)
        for at in range(0, s.shape[-1], 64):
            part = s[..., at:at + 64]
            one = to_bf16((np.abs(part).max(-1, keepdims=True) / np.float32(7.0)).astype(np.float32))
            scale[..., at:at + 64] = np.maximum(one, np.float32(2.0 ** -100))
        q = np.clip(np.rint(s / scale), -7, 7)
        bad = ~(np.abs(s) < np.float32(2.0 ** 102)).all(-1)
        scale[bad] = np.nan
        q[bad] = 0
    return q, scale


def held(x, b):
    """What a cache holds of heads x, in the transformed basis, float64."""
    q, s = quantize(x, b)
    return q.astype(np.float64) * s.astype(np.float64)


def most_scale(x, b):
    """The largest scale of each head, float64."""
    return quantize(x, b)[1].max(-1).astype(np.float64)


class Sequences:
    """A cache of random keys and values: sequences of `lens` in pages dealt at random."""

    def __init__(self, lens, heads, dim, hblock, page, dtype, seed, spare=3, k_scale=1.0, v_scale=1.0, poison=True):
        rng = np.random.default_rng(seed)
        self.lens_np, self.heads, self.dim, self.hblock, self.page = list(lens), heads, dim, hblock, page
        batch = len(self.lens_np)
        width = max(1, -(-max(self.lens_np + [1]) // page))
        pages = batch * width + spare
        self.cache = hatq.hatq_cache4_init(pages, page, heads, dim, hblock=hblock, device=DEV)
        if poison:      # what is not written may hold anything: NaN scales here
            self.cache.buf.fill_(-1)
        self.table_np = rng.permutation(pages)[:batch * width].reshape(batch, width).astype(np.int32)
        self.table, self.lens = dev(self.table_np), dev(np.array(self.lens_np, np.int32))
        total = sum(self.lens_np)
        channel = np.exp(0.5 * rng.normal(size=(2, heads, dim)))
        k = rng.normal(size=(total, heads, dim)) * channel[0] * k_scale
        v = (rng.normal(size=(total, heads, dim)) * channel[1] + 0.3) * v_scale
        self.k, self.v = (torch.from_numpy(x.astype(np.float32)).to(dtype) for x in (k, v))
        self.rng = rng

    def write(self):
        ends = dev(np.cumsum(self.lens_np).astype(np.int32))
        hatq.hatq_cache4_append(self.cache, self.k.to(DEV), self.v.to(DEV), self.table, self.lens, ends=ends)

    def of(self, i):
        """(keys, values) of sequence i as float32 numpy."""
        at = sum(self.lens_np[:i])
        return (x[at:at + self.lens_np[i]].float().numpy() for x in (self.k, self.v))


def attention64(q, k, v, v_scale, hblock, scale, causal, window, fine, there=None):
    """(y, bound) of query rows q [n, q_heads, dim] float32 as the last of the positions of
    keys and values in the transformed basis [len, heads, dim] float64; v_scale [len, heads]:
    the largest of a value's scales; there [len]: positions whose page is.

    The bound (u = 2^-24): the query in two float16 halves is off by 2^-22 = 4 u of itself (many
    rows of bfloat16, in one half, by 2^-11); a product is exact, and a score's sum in float32
    (64 products, two scales of up to four groups, the factor) has at most 80 roundings, u sum
    |q k| each; an error of e moves each normalized weight by at most a factor exp(2 e).  A
    weight times scale in float16 is off by 2^-11 of itself (two halves 2^-21), or where
    subnormal by 2^-25 of a unit that is at most 2 of the largest weight times scale (a value's
    codes may be 0, so the scale and not the value counts); the exponential and the products
    add 8 u.  Float32 sums of len terms add len u each of the magnitudes.  In the end the
    transform's sums add 8 u of the magnitudes."""
    n, heads_q, dim = q.shape
    length, heads = k.shape[:2]
    share = heads_q // heads
    qt = butterfly(q.astype(np.float64), hblock)
    y, bound = np.zeros(q.shape), np.zeros(q.shape)
    factor = scale / hblock
    at, key = length - n + np.arange(n)[:, None], np.arange(length)[None, :]
    keep = np.ones((n, length), bool)
    if causal:
        keep &= key <= at
        if window:
            keep &= key > at - window
    if there is not None:
        keep &= there[None, :]
    rows = keep.any(1)      # of the others all is 0
    if not rows.any():
        return y, bound
    keep, count = keep[rows], keep[rows].sum(1)[:, None]
    for h in range(heads_q):
        # (what no row sees may be anything; what some row does not see is taken out of its sums)
        kk, vv, vs = (np.where(keep.any(0).reshape(-1, *[1] * (x[:, h // share].ndim - 1)), x[:, h // share], 0.0) for x in (k, v, v_scale))
        bad = keep & (np.isnan(kk).any(1) | np.isnan(vv).any(1))[None, :]
        kk, vv, vs = np.nan_to_num(kk, nan=0.0), np.nan_to_num(vv, nan=0.0), np.nan_to_num(vs, nan=0.0)
        qq = qt[rows, h]
        t = np.where(keep, qq @ kk.T * factor, -np.inf)
        e = np.exp(t - t.max(1, keepdims=True))
        w = e / e.sum(1, keepdims=True)
        size = np.where(keep, np.abs(qq) @ np.abs(kk).T, 0.0).max(1, keepdims=True) * abs(factor)
        rel = np.expm1(2 * (80 * U + (2.0 ** -22 if fine else 2.0 ** -11)) * size) + (2.0 ** -21 if fine else 2.0 ** -11)
        rel = rel + (3 * count + 24) * U
        one = butterfly(w @ vv, hblock) / hblock
        low = 2.0 ** -24 * (w * vs[None, :]).max(1, keepdims=True) * 1.01 * 7 * count
        off = rel * butterfly_abs(w @ np.abs(vv), hblock) + low
        one[bad.any(1)] = np.nan
        off[bad.any(1)] = np.nan
        y[rows, h], bound[rows, h] = one, off
    return y, bound


def butterfly_abs(x, b):
    """(1 / b) sum over each block of |x|: what an error of x can move a transform by."""
    s = np.abs(x).reshape(-1, b).sum(1, keepdims=True) / b
    return np.broadcast_to(s, (s.shape[0], b)).reshape(x.shape)


def check(y, y64, bound, what):
    rel, low = ROUND[y.dtype]
    got = y.double().cpu().numpy()
    allowed = bound * (1 + rel) + rel * np.abs(y64) + low
    off = np.where(np.isnan(got) & np.isnan(y64), 0.0, np.abs(got - y64))
    bad = ~((off <= allowed) | (off == 0))
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(off / np.maximum(allowed, 1e-300))} "
                           f"times what is allowed at {np.argwhere(bad)[:4].tolist()}")
