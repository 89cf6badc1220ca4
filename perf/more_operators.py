"""Performance cases of the 4-bit operators: what a decoder that serves tokens reads most
of, its cache of keys and values and its weights, held in 4 bits.

Kinds of case:
  cache    new tokens' keys and values into a paged 4-bit cache (block Hadamard transform
           of each head, codes and a scale for each 64 channels), and read back from it
  attend   queries over that cache: one new token for each sequence, a few, or a part of a
           prompt; grouped heads, causal or not, windows, lengths that differ
  linear4  a few tokens through a linear layer of 4-bit weights with a scale for each
           group of input channels; tokens in INT8 codes, or gated as silu(g) * u

``own`` selects the framework's calls; else ``run`` takes the plain form, elementary torch
operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}
SPAN = 64           # channels of a head that share a scale in the cache


def _cache(name, batch, new, length, heads, dim, hblock, page, dtype, ragged=False, strided=False):
    """`new` tokens at the end of each sequence, which then has `length`."""
    c = {"kind": "cache", "batch": batch, "new": new, "length": length, "heads": heads, "dim": dim, "hblock": hblock,
         "page": page, "dtype": dtype, "ragged": ragged, "strided": strided}
    return {"name": name, **c} if name else c


def _attend(name, batch, new, length, q_heads, heads, dim, hblock, page, dtype, spread=0.0, ragged=False, causal=True,
            window=0):
    """Sequences of `length` down to (1 - spread) of it, the last `new` tokens asking."""
    c = {"kind": "attend", "batch": batch, "new": new, "length": length, "q_heads": q_heads, "heads": heads, "dim": dim,
         "hblock": hblock, "page": page, "dtype": dtype, "spread": spread, "ragged": ragged, "causal": causal,
         "window": window}
    return {"name": name, **c} if name else c


def _linear4(name, rows, cin, cout, dtype, hblock, group, bias=False, gated=False, strided=False):
    """gated: the layer holds 2 * cout channels and gives cout."""
    c = {"kind": "linear4", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "hblock": hblock, "group": group,
         "bias": bias, "gated": gated, "strided": strided}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one step of a few sequences: launches and host work
        _cache("cache_step", 8, 1, 500, 8, 128, 128, 64, "bf16"),
        # odd head size and page, float32, ragged
        _cache("cache_odd", 5, 77, 300, 3, 80, 16, 16, "fp32", ragged=True),
        # a batch of prompts, keys and values inside the rows of a query-key-value product
        _cache("cache_prompt", 4, 8192, 8192, 8, 128, 128, 64, "bf16", strided=True),
        # one sequence, one token, a short context, as many key as query heads: latency
        _attend("attend_small", 1, 1, 300, 8, 8, 64, 64, 16, "bf16"),
        # a serving batch's step, lengths that differ
        _attend("attend_step", 32, 1, 4096, 32, 8, 128, 128, 64, "bf16", spread=0.8),
        # two long documents, float16
        _attend("attend_long", 2, 1, 131072, 32, 4, 128, 64, 256, "fp16"),
        # a large batch's step: the largest in bytes
        _attend("attend_batch", 64, 1, 16384, 64, 8, 128, 128, 64, "bf16", spread=0.1),
        # a few tokens to verify for each sequence, odd sizes, a window, float32
        _attend("attend_few", 7, 5, 1500, 12, 4, 80, 16, 16, "fp32", spread=0.5, window=700),
        # parts of prompts, ragged: the largest in operations
        _attend("attend_prompt", 3, 2048, 8192, 16, 2, 128, 128, 64, "bf16", spread=0.5, ragged=True),
        # one token through a square layer of a decoder: launches and the weights' bytes
        _linear4("linear4_token", 1, 4096, 4096, "bf16", 128, 128),
        # a few sequences, the gated half of a large feed-forward block
        _linear4("linear4_gated", 6, 8192, 16384, "bf16", 64, 64, gated=True),
        # odd widths out of a wider buffer, float32, past a few tokens
        _linear4("linear4_odd", 77, 1000, 1001, "fp32", 8, 64, bias=True, strided=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _blocks(rng, width):
    return rng.choice([b for b in (1, 8, 16, 32, 64, 64, 128, 128) if width % b == 0])


def draw(rng):
    while True:
        kind = rng.choice(["cache", "attend", "attend", "linear4"])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        page = rng.choice([16, 32, 64, 64, 256])
        dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 192, 256])
        if kind == "cache":
            new = _log(rng, 1, 8192)
            c = _cache(None, _log(rng, 1, 64), new, new + rng.randint(0, 500), _log(rng, 1, 16), dim, _blocks(rng, dim),
                       page, dtype, ragged=rng.random() < 0.5, strided=rng.random() < 0.3)
            if c["batch"] * c["new"] * c["heads"] * dim > 2e7:
                continue
        elif kind == "attend":
            heads, new = rng.choice([1, 2, 3, 4, 8, 8]), rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 2048)])
            length = _log(rng, max(1, new), 131072)
            causal = rng.random() < 0.8
            c = _attend(None, _log(rng, 1, 64), new, length, heads * rng.choice([1, 2, 4, 5, 8]), heads, dim,
                        _blocks(rng, dim), page, dtype, spread=rng.choice([0.0, 0.1, 0.5, 0.9]),
                        ragged=rng.random() < 0.3, causal=causal,
                        window=_log(rng, 1, 8192) if causal and rng.random() < 0.2 else 0)
            pairs = c["batch"] * float(new) * length * c["q_heads"]
            if c["batch"] * length * heads * dim > 3e8 or pairs > 2e8 or pairs * dim > 2e10:
                continue
        else:
            group = rng.choice([64, 128])
            hblock = rng.choice([1, 8, 64, 64, 128, 128])
            c = _linear4(None, _log(rng, 1, 128), max(1, _log(rng, 64, 16384) // hblock) * hblock, _log(rng, 16, 16384),
                         dtype, hblock, group, bias=rng.random() < 0.5, gated=rng.random() < 0.3,
                         strided=rng.random() < 0.3)
            if c["cin"] * c["cout"] * (2 if c["gated"] else 1) > 1.4e8 or c["rows"] * c["cin"] * c["cout"] > 2e9:
                continue
        return c


# ---- what a case holds ---------------------------------------------------------

def _lengths(c):
    """Each sequence's length, its new tokens among them."""
    if c["kind"] == "cache":
        return [c["length"]] * c["batch"]
    return [max(1, int(c["length"] * (1.0 - c["spread"] * ((5 * b + 3) % c["batch"]) / c["batch"])))
            for b in range(c["batch"])]


def _new(c):
    """Each sequence's new tokens."""
    lens = _lengths(c)
    if not c["ragged"]:
        return [min([c["new"]] + lens)] * c["batch"]
    return [max(1, min(n, c["new"] * ((3 * b + 1) % c["batch"] + 1) // c["batch"])) for b, n in enumerate(lens)]


def _visible(c):
    """Pairs of a new token and a position that it sees, of all sequences."""
    total = 0.0
    for length, new in zip(_lengths(c), _new(c)):
        for i in range(new):
            seen = length - new + i + 1 if c["causal"] else length
            total += min(seen, c["window"]) if c["window"] else seen
    return total


# ---- inputs ------------------------------------------------------------------

def _features(gen, rows, heads, dim, mean=2.0):
    """Keys or values: a scale for each channel, a few channels with a large mean."""
    scale = torch.exp(0.5 * torch.randn(heads, dim, generator=gen, device=DEV))
    x = torch.randn(rows, heads, dim, generator=gen, device=DEV)
    x *= scale
    shift = torch.randint(0, dim, (2,), generator=gen, device=DEV)
    x[:, :, shift] += mean * scale[:, shift]
    return x


def _tokens(gen, rows, cin, dtype, strided=False):
    """Activations: per-channel log-normal scales, a heavy tail, a few channels with a
    large mean."""
    scale = torch.exp(0.7 * torch.randn(cin, generator=gen, device=DEV))
    x = torch.randn(rows, cin, generator=gen, device=DEV)
    x = x * (1.0 + 0.1 * x * x) * scale
    shift = torch.randint(0, cin, (min(8, cin),), generator=gen, device=DEV)
    x[:, shift] += 3.0 * scale[shift]
    x = x.to(DTYPES[dtype])
    if strided:
        wide = torch.zeros(rows, cin + 24, dtype=x.dtype, device=DEV)
        wide[:, 8:8 + cin] = x
        x = wide[:, 8:8 + cin]
    return x


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["kind"] == "linear4":
        held = case["cout"] * (2 if case["gated"] else 1)
        cin, groups = case["cin"], -(-case["cin"] // case["group"])
        # a quantized checkpoint: codes, a scale for each channel and group, a bias
        codes = torch.randn(held, cin, generator=gen, device=DEV).mul_(2.5).round_().clamp_(-7, 7).to(torch.int8)
        scale = torch.rand(held, groups, generator=gen, device=DEV).add_(0.5).mul_(1.0 / (2.5 * math.sqrt(cin)))
        bias = torch.randn(held, generator=gen, device=DEV).mul_(0.1) if case["bias"] else None
        return {"x": _tokens(gen, case["rows"], cin, case["dtype"], case["strided"]),
                "layer": (codes, scale.to(torch.bfloat16), bias)}
    lens, new, dtype = _lengths(case), _new(case), DTYPES[case["dtype"]]
    width = -(-max(lens) // case["page"])
    pages = case["batch"] * width
    s = {"lens": _ints(lens), "pages": pages,
         "table": torch.randperm(pages, generator=gen, device=DEV).to(torch.int32).view(case["batch"], width)}
    # the rows' ends, where sequences have unlike numbers of new tokens
    s["ends"] = torch.cumsum(_ints(new), 0).to(torch.int32) if case["ragged"] else None
    rows, heads, dim = sum(new), case["heads"], case["dim"]
    if case["kind"] == "cache":
        k, v = _features(gen, rows, heads, dim), _features(gen, rows, heads, dim, 0.5)
        if case["strided"]:
            wide = torch.zeros(rows, 6 * heads, dim, dtype=dtype, device=DEV)
            wide[:, 4 * heads:5 * heads], wide[:, 5 * heads:] = k, v
            k, v = wide[:, 4 * heads:5 * heads], wide[:, 5 * heads:]
        return {**s, "k": k.to(dtype), "v": v.to(dtype)}
    k = _features(gen, sum(lens), heads, dim).to(dtype)
    v = _features(gen, sum(lens), heads, dim, 0.5).to(dtype)
    q = torch.randn(rows, case["q_heads"], dim, generator=gen, device=DEV)
    return {**s, "k": k, "v": v, "q": q.to(dtype), "k_ends": torch.cumsum(_ints(lens), 0).to(torch.int32)}


def _places(table, page, first, count):
    """Of the rows of all sequences in turn, `count[b]` of them from position first[b] on:
    each row's page and its place in the page."""
    seq = torch.repeat_interleave(torch.arange(len(count), device=DEV), count)
    begin = torch.cumsum(count, 0) - count
    pos = torch.arange(seq.shape[0], device=DEV) - begin[seq] + first[seq]
    return table[seq, pos // page].long(), pos % page


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "linear4":
        if own:
            from paper_2608_01653_amd import hatq
            codes, scale, bias = s.pop("layer")
            s["lin"] = hatq.hatq_pack_linear4(codes, scale, bias=bias, hblock=case["hblock"], gated=case["gated"])
            s["forward"] = hatq.hatq_linear4_forward
        return s
    heads, dim, pages, page = case["heads"], case["dim"], s.pop("pages"), case["page"]
    if own:
        from paper_2608_01653_amd import hatq
        s["hatq"] = hatq
        s["cache"] = hatq.hatq_cache4_init(pages, page, heads, dim, hblock=case["hblock"], device=DEV)
        if case["kind"] == "attend":
            # the context, as earlier steps have written it
            hatq.hatq_cache4_append(s["cache"], s.pop("k"), s.pop("v"), s["table"], s["lens"], ends=s.pop("k_ends"))
        return s
    groups = -(-dim // SPAN)
    for x in ("k", "v"):
        s[x + "_codes"] = torch.zeros(pages, page, heads, dim, dtype=torch.int8, device=DEV)
        s[x + "_scale"] = torch.zeros(pages, page, heads, groups, dtype=torch.bfloat16, device=DEV)
    if case["kind"] == "attend":
        s.pop("k_ends")
        at = _places(s["table"], page, torch.zeros_like(s["lens"]).long(), s["lens"].long())
        for x in ("k", "v"):
            s[x + "_codes"][at], s[x + "_scale"][at] = _quantize4(s.pop(x), case["hblock"])
    # the rows of each sequence, which a plain program plans its padding by
    s["most"], s["rows"] = max(_new(case)), sum(_new(case))
    return s


# ---- the plain form ----------------------------------------------------------

def _butterfly(x, hblock):
    """Unnormalized Sylvester transform of each block of `hblock` channels."""
    shape, h = x.shape, 1
    while h < hblock:
        v = x.reshape(-1, 2, h)
        x = torch.stack((v[:, 0] + v[:, 1], v[:, 0] - v[:, 1]), 1)
        h *= 2
    return x.reshape(shape)


def _per_channel(scale, dim):
    """The scale of each channel from those of its groups."""
    return torch.repeat_interleave(scale, SPAN, dim=-1)[..., :dim]


def _quantize4(x, hblock):
    """Heads [..., dim]: codes, and a scale for each 64 channels."""
    dim = x.shape[-1]
    v = _butterfly(x.float(), hblock)
    wide = torch.nn.functional.pad(v, (0, -dim % SPAN)).unflatten(-1, (-1, SPAN))
    most = wide.abs().amax(-1)
    scale = (most / torch.full_like(most, 7.0)).to(torch.bfloat16)  # a division: by a number, torch multiplies
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return torch.round(v / _per_channel(scale.float(), dim)).clamp(-7.0, 7.0).to(torch.int8), scale


def _new_count(s):
    case = s["case"]
    if s["ends"] is None:
        return torch.full_like(s["lens"], s["rows"] // case["batch"]).long()
    return torch.diff(s["ends"], prepend=s["ends"].new_zeros(1)).long()


def _plain_cache(s):
    case = s["case"]
    count = _new_count(s)
    at = _places(s["table"], case["page"], s["lens"].long() - count, count)
    out = []
    for x in ("k", "v"):
        s[x + "_codes"][at], s[x + "_scale"][at] = _quantize4(s[x], case["hblock"])
        values = s[x + "_codes"][at].float() * _per_channel(s[x + "_scale"][at].float(), case["dim"])
        out.append((_butterfly(values, case["hblock"]) * (1.0 / case["hblock"])).to(s[x].dtype))
    return tuple(out)


def _paged(s, x):
    """[batch, heads, positions, dim], transformed values of the cache's pages."""
    table, dim = s["table"].long(), s["case"]["dim"]
    values = s[x + "_codes"][table].flatten(1, 2).transpose(1, 2).float()
    return values.mul_(_per_channel(s[x + "_scale"][table].flatten(1, 2).transpose(1, 2).float(), dim))


def _plain_attend(s):
    case, lens = s["case"], s["lens"].long()
    batch, heads, dim, most = case["batch"], case["heads"], case["dim"], s["most"]
    count = _new_count(s)
    i = torch.arange(most, device=DEV)
    there = i[None, :] < count[:, None]
    row = ((torch.cumsum(count, 0) - count)[:, None] + i[None, :]).clamp(max=s["rows"] - 1)
    q = _butterfly(s["q"].float(), case["hblock"])[row]                       # [batch, most, q_heads, dim]
    q = q.view(batch, most, heads, -1, dim).permute(0, 2, 1, 3, 4).reshape(batch, heads, -1, dim)
    # a head holds b times the original products after both transforms
    score = torch.matmul(q, _paged(s, "k").transpose(2, 3)) * (1.0 / (case["hblock"] * math.sqrt(dim)))
    score = score.view(batch, heads, most, -1, score.shape[-1])
    key = torch.arange(score.shape[-1], device=DEV)
    seen = (key[None, :] < lens[:, None])[:, None, :]
    if case["causal"]:
        at = (lens - count)[:, None] + i[None, :]
        seen = seen & (key <= at[:, :, None])
        if case["window"]:
            seen = seen & (key > at[:, :, None] - case["window"])
    score = score.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    p = p.flatten(2, 3)
    y = torch.matmul(p, _paged(s, "v")).view(batch, heads, most, -1, dim) / torch.where(total == 0, torch.ones_like(total), total)
    y = y.permute(0, 2, 1, 3, 4).reshape(batch, most, -1, dim)[there]
    return (_butterfly(y, case["hblock"]) * (1.0 / case["hblock"])).to(s["q"].dtype)


def _plain_linear4(s):
    case, x = s["case"], s["x"]
    codes, w_scale, bias = s["layer"]
    v = _butterfly(x.float(), case["hblock"])
    most = v.abs().amax(1, keepdim=True)
    scale = most / torch.full_like(most, 127.0)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    q = torch.round(v / scale).clamp(-127.0, 127.0)
    w = codes.float() * torch.repeat_interleave(w_scale.float(), case["group"], dim=1)[:, :case["cin"]]
    y = (q @ w.t()) * (scale * (1.0 / case["hblock"]))
    if bias is not None:
        y = y + bias
    if case["gated"]:
        g, u = y.chunk(2, dim=-1)
        y = g / (1.0 + torch.exp(-g)) * u
    return y.to(x.dtype)


def run(state):
    case = state["case"]
    if not own:
        return {"cache": _plain_cache, "attend": _plain_attend, "linear4": _plain_linear4}[case["kind"]](state)
    if case["kind"] == "linear4":
        return state["forward"](state["lin"], state["x"])
    hatq, cache, place = state["hatq"], state["cache"], (state["table"], state["lens"])
    if case["kind"] == "cache":
        hatq.hatq_cache4_append(cache, state["k"], state["v"], *place, ends=state["ends"])
        return hatq.hatq_cache4_read(cache, state["k"].shape[0], *place, ends=state["ends"], out_dtype=state["k"].dtype)
    return hatq.hatq_attention4(cache, state["q"], *place, ends=state["ends"], causal=case["causal"],
                                window=case["window"])


# ---- what a pass cannot do without ---------------------------------------------

def work(case):
    size = SIZES[case["dtype"]]
    if case["kind"] == "linear4":
        held = case["cout"] * (2 if case["gated"] else 1)
        data = case["rows"] * (case["cin"] + case["cout"]) * size
        weights = held * (0.5 * case["cin"] + 2 * -(-case["cin"] // case["group"]) + (4 if case["bias"] else 0))
        return {"bytes": data + weights, "flops": 2.0 * case["rows"] * case["cin"] * held}
    rows, dim = sum(_new(case)), case["dim"]
    held = case["heads"] * (dim + 4.0 * -(-dim // SPAN))        # a position's codes and scales, keys and values
    if case["kind"] == "cache":
        # written by one call and read by the next
        stages = max(0, case["hblock"].bit_length() - 1)
        return {"bytes": rows * (4.0 * case["heads"] * dim * size + 2 * held),
                "flops": rows * case["heads"] * dim * 2.0 * (2 * stages + 4)}
    met = 0.0
    for length, new in zip(_lengths(case), _new(case)):
        met += min(length, case["window"] + new - 1) if case["window"] else length
    return {"bytes": met * held + 2.0 * rows * case["q_heads"] * dim * size,
            "flops": 4.0 * dim * case["q_heads"] * _visible(case)}


# ---- the definition in 64 bits -------------------------------------------------

def _sylvester(order):
    i = torch.arange(order, device=DEV)
    both, odd = i[:, None] & i[None, :], torch.zeros(order, order, dtype=torch.long, device=DEV)
    for bit in range(8):
        odd ^= (both >> bit) & 1
    return 1.0 - 2.0 * odd.double()


def _transform64(x, hblock):
    return (x.reshape(-1, hblock) @ _sylvester(hblock)).reshape(x.shape)


def _stages32(x, hblock):
    """The transform that codes are made of: by definition float32 sums, stage by stage."""
    i, x = torch.arange(x.shape[-1], device=DEV), x.float()
    for bit in range(hblock.bit_length() - 1):
        other = x[..., i ^ (1 << bit)]
        x = torch.where((i >> bit) % 2 == 1, other - x, x + other)
    return x.double()


def _codes64(part, step, most):
    """Whole numbers next to S / step, the quotient a float32 as the definition has it."""
    return torch.clamp(torch.round((part / step).float()), -most, most).double()


def _exact_codes(x, hblock):
    """The values that 4-bit codes of heads x stand for, in the transformed basis."""
    v = _stages32(x, hblock)
    out = torch.empty_like(v)
    for at in range(0, v.shape[-1], SPAN):
        part = v[..., at:at + SPAN]
        step = (part.abs().amax(-1, keepdim=True) / 7.0).float().to(torch.bfloat16).double()
        step[step == 0] = 1.0
        out[..., at:at + SPAN] = _codes64(part, step, 7) * step
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    hblock = case["hblock"]
    if case["kind"] == "cache":
        return tuple(_transform64(_exact_codes(s[x], hblock), hblock) / hblock for x in ("k", "v"))
    if case["kind"] == "linear4":
        codes, w_scale, bias = s["layer"]
        t = _stages32(s["x"], hblock)
        step = (t.abs().amax(dim=1, keepdim=True) / 127.0).float().double()
        step[step == 0] = 1.0
        q, z = _codes64(t, step, 127), 0.0
        for g in range(w_scale.shape[1]):
            part = slice(g * case["group"], (g + 1) * case["group"])
            z = z + (q[:, part] @ codes[:, part].double().T.contiguous()) * w_scale[:, g].double()
        z = z * step / hblock
        if bias is not None:
            z = z + bias.double()
        if case["gated"]:
            half = z.shape[1] // 2
            z = z[:, :half] * torch.sigmoid(z[:, :half]) * z[:, half:]
        return z
    out, at, row = [], 0, 0
    share = case["q_heads"] // case["heads"]
    for length, new in zip(_lengths(case), _new(case)):
        k, v = (_exact_codes(s[x][at:at + length], hblock) for x in ("k", "v"))
        q = _transform64(s["q"][row:row + new].double(), hblock)
        at, row = at + length, row + new
        here = torch.arange(length - new, length, device=DEV)[:, None]
        key = torch.arange(length, device=DEV)[None, :]
        hidden = torch.zeros(new, length, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= key > here
        if case["window"]:
            hidden |= key <= here - case["window"]
        y = torch.empty_like(q)
        for h in range(case["q_heads"]):
            score = q[:, h] @ k[:, h // share].T.contiguous() / (hblock * math.sqrt(case["dim"]))
            y[:, h] = torch.softmax(score.masked_fill_(hidden, float("-inf")), dim=-1) @ v[:, h // share].contiguous()
        out.append(_transform64(y, hblock) / hblock)
    return torch.cat(out)
