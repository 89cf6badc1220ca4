"""Performance cases of the INT8 linear layers over tokens: what a transformer's linear
layers, expert layers and gated feed-forward blocks have the library do.

Kinds of case:
  linear   tokens [rows, cin] through one INT8 layer: block Hadamard transform and a
           scale for each token, INT8 product with a scale for each channel, bias, or the
           gated unit silu(g) * u of a layer that holds both halves
  experts  rows grouped by expert, ragged, gathered from their tokens, each group through
           its expert's INT8 layer
  moe      a feed-forward block of gated experts: chosen experts and their weights for
           each token, both expert layers, the weighted sum

``own`` selects the framework's calls; else ``run`` takes the plain form, elementary torch
operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}

# the work of the largest listed case, in INT8 operations; draws stay below it
MOST_OPS = 1.1e12


def _linear(name, rows, cin, cout, dtype, hblock, bias=False, gated=False, strided=False):
    """gated: the layer holds 2 * cout channels and gives cout."""
    c = {"kind": "linear", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "hblock": hblock,
         "bias": bias, "gated": gated, "strided": strided}
    return {"name": name, **c} if name else c


def _experts(name, tokens, topk, experts, cin, cout, dtype, hblock, bias=False, gated=False):
    c = {"kind": "experts", "tokens": tokens, "topk": topk, "experts": experts, "cin": cin, "cout": cout,
         "dtype": dtype, "hblock": hblock, "bias": bias, "gated": gated}
    return {"name": name, **c} if name else c


def _moe(name, tokens, topk, experts, width, hidden, dtype, hblock):
    c = {"kind": "moe", "tokens": tokens, "topk": topk, "experts": experts, "width": width, "hidden": hidden,
         "dtype": dtype, "hblock": hblock}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of an entropy model, widths of a codec's latents: launches and host work
        _linear("token_small", 1, 320, 192, "bf16", 64, bias=True),
        # one token through a square layer of a decoder: the weights' bytes
        _linear("token", 1, 4096, 4096, "bf16", 128),
        # a few sequences decoding, the gated half of a feed-forward block
        _linear("tokens_gated", 13, 4096, 8192, "fp16", 128, gated=True),
        # odd widths out of a wider buffer, float32
        _linear("batch_odd", 77, 1000, 1001, "fp32", 8, bias=True, strided=True),
        # the latents of a 1024x1536 image as tokens, float32 as the codec keeps them
        _linear("latents", 6144, 320, 320, "fp32", 64, bias=True),
        # a prompt through a square layer
        _linear("prompt", 4096, 4096, 4096, "bf16", 128),
        # a long prompt through the gated half of a feed-forward block: the largest
        _linear("prompt_gated", 8192, 4096, 8192, "bf16", 64, gated=True),
        # a few sequences decoding over many experts: most experts have no row or one
        _experts("experts_tokens", 12, 4, 64, 2048, 1024, "bf16", 128),
        # an odd number of tokens, no transform, a bias for each expert
        _experts("experts_odd", 1367, 3, 16, 1024, 2048, "fp16", 1, bias=True),
        # a batch of prompts
        _experts("experts_prompt", 8192, 4, 64, 2048, 1024, "bf16", 128, gated=True),
        # the whole block for a few sequences, and for a prompt
        _moe("moe_tokens", 24, 4, 32, 1024, 512, "bf16", 64),
        _moe("moe_prompt", 4096, 4, 32, 2048, 1024, "bf16", 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ops(c):
    if c["kind"] == "linear":
        return 2.0 * c["rows"] * c["cin"] * c["cout"] * (2 if c["gated"] else 1)
    pairs = c["tokens"] * c["topk"]
    if c["kind"] == "experts":
        return 2.0 * pairs * c["cin"] * c["cout"] * (2 if c["gated"] else 1)
    return 2.0 * pairs * c["width"] * c["hidden"] * 3


def draw(rng):
    while True:
        kind = rng.choice(["linear", "linear", "experts", "moe"])
        # (a moe block quantizes what it has computed: a last bit there moves a code now and
        # then, which is below what 16-bit outputs hold and above what float32 ones do)
        dtype = rng.choice(["bf16", "bf16", "fp16", "bf16" if kind == "moe" else "fp32"])
        hblock = rng.choice([1, 8, 64, 64, 128, 128])
        if kind == "linear":
            c = _linear(None, _log(rng, 1, 8192), max(1, _log(rng, 64, 8192) // hblock) * hblock, _log(rng, 16, 8192),
                        dtype, hblock, bias=rng.random() < 0.5, gated=rng.random() < 0.3,
                        strided=rng.random() < 0.3)
        elif kind == "experts":
            experts = _log(rng, 2, 64)
            c = _experts(None, _log(rng, 1, 8192), rng.randint(1, min(6, experts)), experts,
                         max(1, _log(rng, 128, 4096) // hblock) * hblock, _log(rng, 64, 4096), dtype, hblock,
                         bias=rng.random() < 0.3, gated=rng.random() < 0.3)
            if experts * c["cin"] * c["cout"] > 3e8:
                continue
        else:
            experts = _log(rng, 4, 64)
            c = _moe(None, _log(rng, 1, 4096), rng.randint(1, min(6, experts)), experts,
                     max(1, _log(rng, 128, 2048) // hblock) * hblock, max(1, _log(rng, 64, 2048) // hblock) * hblock,
                     dtype, hblock)
            if experts * c["width"] * c["hidden"] > 1e8:
                continue
        if _ops(c) <= MOST_OPS * 0.3:
            return c


# ---- inputs ------------------------------------------------------------------

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


def _layer(gen, experts, cout, cin, bias):
    """A quantized checkpoint: codes [experts, cout, cin], a scale for each channel, a bias."""
    codes = torch.randn(experts, cout, cin, generator=gen, device=DEV).mul_(30.0).round_().clamp_(-127, 127)
    codes = codes.to(torch.int8)
    scale = torch.rand(experts, cout, generator=gen, device=DEV).add_(0.5).mul_(1.0 / (30.0 * math.sqrt(cin)))
    b = torch.randn(experts, cout, generator=gen, device=DEV).mul_(0.1) if bias else None
    return codes, scale, b


def _chosen(gen, tokens, topk, experts):
    """Each token's experts and their weights, some experts more popular than others."""
    score = torch.randn(tokens, experts, generator=gen, device=DEV)
    score = score + 0.5 * torch.randn(experts, generator=gen, device=DEV)
    top, ids = torch.topk(score, topk, dim=1)
    return ids.to(torch.int32), torch.softmax(top, dim=1)


def _grouping(ids, experts):
    """Row ends of each expert, and the token of each row, for rows sorted by expert."""
    flat = ids.reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    ends = torch.cumsum(torch.bincount(flat, minlength=experts), 0).to(torch.int32)
    return ends, (order // ids.shape[1]).to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    g = 2 if case.get("gated") else 1
    if case["kind"] == "linear":
        return {"x": _tokens(gen, case["rows"], case["cin"], case["dtype"], case["strided"]),
                "layer": _layer(gen, 1, g * case["cout"], case["cin"], case["bias"])}
    ids, weights = _chosen(gen, case["tokens"], case["topk"], case["experts"])
    if case["kind"] == "experts":
        ends, src = _grouping(ids, case["experts"])
        return {"x": _tokens(gen, case["tokens"], case["cin"], case["dtype"]), "ends": ends, "src": src,
                "layer": _layer(gen, case["experts"], g * case["cout"], case["cin"], case["bias"])}
    return {"x": _tokens(gen, case["tokens"], case["width"], case["dtype"]), "ids": ids, "weights": weights,
            "in": _layer(gen, case["experts"], 2 * case["hidden"], case["width"], False),
            "out": _layer(gen, case["experts"], case["width"], case["hidden"], False)}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        # the layers laid out once, as a program does with its checkpoint
        from paper_2608_01653_amd import experts, hatq

        def pack(layer, gated):
            codes, scale, bias = layer
            return hatq.hatq_pack_linear(codes, scale, bias=bias, hblock=case["hblock"], gated=gated)

        if case["kind"] == "moe":
            s["mlp"] = experts.ExpertMLP(pack(s.pop("in"), True), pack(s.pop("out"), False))
        else:
            s["lin"] = pack(s.pop("layer"), case["gated"])
            s["forward"] = hatq.hatq_linear_forward if case["kind"] == "linear" else hatq.hatq_experts_forward
    elif case["kind"] != "linear":
        # the largest group, which a plain program reads back once when it plans its padding
        ends = s["ends"] if "ends" in s else _grouping(s["ids"], case["experts"])[0]
        s["most"] = int(torch.diff(ends, prepend=ends.new_zeros(1)).max())
    return s


# ---- the plain form ----------------------------------------------------------

def _butterfly(x, hblock):
    """Unnormalized Sylvester transform of each block of `hblock` channels."""
    rows, h = x.shape[0], 1
    while h < hblock:
        v = x.view(rows, -1, 2, h)
        x = torch.stack((v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]), 2)
        h *= 2
    return x.reshape(rows, -1)


def _quantize(x, hblock):
    """Codes, as float32, and the scale of each token."""
    v = _butterfly(x.float().contiguous(), hblock)
    most = v.abs().amax(1, keepdim=True)
    scale = most / torch.full_like(most, 127.0)     # a division: by a number, torch multiplies by 1 / 127
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return torch.round(v / scale).clamp(-127.0, 127.0), scale


def _finish(acc, scale, w_scale, bias, hblock, gated):
    y = acc * (scale * w_scale * (1.0 / hblock))
    if bias is not None:
        y = y + bias
    if gated:
        g, u = y.chunk(2, dim=-1)
        y = g / (1.0 + torch.exp(-g)) * u
    return y


def _plain_linear(x, layer, hblock, gated):
    codes, w_scale, bias = layer
    q, scale = _quantize(x, hblock)
    acc = q @ codes[0].float().t()
    return _finish(acc, scale, w_scale[0], None if bias is None else bias[0], hblock, gated)


def _plain_grouped(q, scale, layer, ends, most, hblock, gated):
    """Rows sorted by expert: each group padded to the largest, one batched product."""
    codes, w_scale, bias = layer
    experts, _, cin = codes.shape
    row = torch.arange(q.shape[0], device=q.device)
    expert = torch.searchsorted(ends.long(), row, right=True)
    begin = torch.cat((ends.new_zeros(1), ends[:-1])).long()
    padded = q.new_zeros(experts, most, cin)
    padded[expert, row - begin[expert]] = q
    acc = torch.bmm(padded, codes.float().transpose(1, 2).contiguous())[expert, row - begin[expert]]
    return _finish(acc, scale, w_scale[expert], None if bias is None else bias[expert], hblock, gated)


def _plain(s):
    case, x = s["case"], s["x"]
    hblock = case["hblock"]
    if case["kind"] == "linear":
        return _plain_linear(x, s["layer"], hblock, case["gated"]).to(x.dtype)
    if case["kind"] == "experts":
        q, scale = _quantize(x, hblock)
        src = s["src"].long()
        return _plain_grouped(q[src], scale[src], s["layer"], s["ends"], s["most"], hblock, case["gated"]).to(x.dtype)
    flat = s["ids"].reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    ends = torch.cumsum(torch.bincount(flat, minlength=case["experts"]), 0)
    q, scale = _quantize(x, hblock)
    src = order // case["topk"]
    hidden = _plain_grouped(q[src], scale[src], s["in"], ends, s["most"], hblock, True)
    q, scale = _quantize(hidden, hblock)
    rows = _plain_grouped(q, scale, s["out"], ends, s["most"], hblock, False)
    back = torch.empty_like(rows)
    back[order] = rows
    back = back.view(case["tokens"], case["topk"], -1)
    return (back * s["weights"][:, :, None]).sum(1).to(x.dtype)


def run(state):
    if not own:
        return _plain(state)
    case = state["case"]
    if case["kind"] == "linear":
        return state["forward"](state["lin"], state["x"])
    if case["kind"] == "experts":
        return state["forward"](state["lin"], state["x"], state["ends"], src=state["src"])
    return state["mlp"](state["x"], state["ids"], state["weights"])


# ---- what a pass cannot do without ---------------------------------------------

def work(case):
    size = SIZES[case["dtype"]]
    if case["kind"] == "linear":
        held = case["cout"] * (2 if case["gated"] else 1)
        data = case["rows"] * (case["cin"] + case["cout"]) * size
        weights = held * (case["cin"] + 4 + (4 if case["bias"] else 0))
        return {"bytes": data + weights, "flops": _ops(case)}
    pairs, experts = case["tokens"] * case["topk"], case["experts"]
    met = experts * (1.0 - (1.0 - 1.0 / experts) ** pairs)      # experts that have a row
    if case["kind"] == "experts":
        held = case["cout"] * (2 if case["gated"] else 1)
        data = (case["tokens"] * case["cin"] + pairs * case["cout"]) * size + 4 * pairs + 4 * experts
        weights = met * held * (case["cin"] + 4 + (4 if case["bias"] else 0))
    else:
        data = 2 * case["tokens"] * case["width"] * size + 8 * pairs
        weights = met * (3 * case["hidden"] * case["width"] + 8 * case["hidden"] + 4 * case["width"])
    return {"bytes": data + weights, "flops": _ops(case)}


# ---- the definition in 64 bits -------------------------------------------------

def _sylvester(order):
    i = torch.arange(order, device=DEV)
    both, odd = i[:, None] & i[None, :], torch.zeros(order, order, dtype=torch.long, device=DEV)
    for bit in range(8):
        odd ^= (both >> bit) & 1
    return 1.0 - 2.0 * odd.double()


def _exact_layer(x, codes, w_scale, bias, hblock, gated):
    """Each row of x (64 bits) through the layer of its expert."""
    s = (x.reshape(x.shape[0], -1, hblock) @ _sylvester(hblock)).reshape(x.shape)
    step = s.abs().amax(dim=1) / 127.0
    step = torch.where(step > 0, step, torch.ones_like(step))[:, None]
    q = torch.clamp(torch.round(s / step), -127, 127)
    z = (q @ codes.double().T.contiguous()) * step * w_scale.double() / hblock
    if bias is not None:
        z = z + bias.double()
    if gated:
        half = z.shape[1] // 2
        z = z[:, :half] * torch.sigmoid(z[:, :half]) * z[:, half:]
    return z


def _exact_groups(rows, layer, ends, hblock, gated):
    codes, w_scale, bias = layer
    out, begin = [], 0
    for e, end in enumerate(ends.tolist()):
        if end > begin:
            out.append(_exact_layer(rows[begin:end], codes[e], w_scale[e], None if bias is None else bias[e],
                                    hblock, gated))
        begin = end
    return torch.cat(out)


def exact(case, seed):
    s = _inputs(case, seed)
    x, hblock = s["x"].double(), case["hblock"]
    if case["kind"] == "linear":
        codes, w_scale, bias = s["layer"]
        return _exact_layer(x, codes[0], w_scale[0], None if bias is None else bias[0], hblock, case["gated"])
    if case["kind"] == "experts":
        return _exact_groups(x[s["src"].long()], s["layer"], s["ends"], hblock, case["gated"])
    ends, src = _grouping(s["ids"], case["experts"])
    hidden = _exact_groups(x[src.long()], s["in"], ends, hblock, True)
    rows = _exact_groups(hidden, s["out"], ends, hblock, False)
    place = torch.argsort(torch.argsort(s["ids"].reshape(-1).long(), stable=True))   # the row of each pair
    picked = rows[place].reshape(case["tokens"], case["topk"], -1)
    return (s["weights"].double()[:, :, None] * picked).sum(1)
