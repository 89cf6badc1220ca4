"""The expert block in one call against its steps called one by one, bit for bit: every
instance of its first launch (the rows' order beside the tokens' codes), its fallbacks,
both layouts of its workspace (output rows beside the hidden rows, and in their place), in
a workspace of exactly the size asked for with guard bytes around it.  The steps have
tests of their own against 64 bits.

test_linear_choice.py shows on the CPU that BLOCKS holds both layouts and every instance.
"""
import numpy as np
import pytest
import torch

from gpu_util import DEV, Guarded, dev
from paper_2608_01653_amd import experts, hatq

pytestmark = pytest.mark.gpu

# tokens, topk, experts, width, hidden, block of the transform
BLOCKS = [
    # a wave a row of one and two chunks, 2, 4 and 8 waves a row: token counts that leave the
    # last block part of its rows, one token
    (1, 2, 4, 448, 64, 64), (13, 3, 6, 512, 192, 64), (9, 2, 5, 700, 260, 4), (1025, 2, 3, 1024, 320, 64), (7, 2, 4, 1088, 64, 64),
    (203, 4, 7, 2048, 128, 128), (1, 1, 1, 2112, 96, 32), (3, 6, 8, 4096, 256, 128), (5, 2, 3, 4160, 64, 64), (1, 4, 6, 8192, 128, 128),
    (33, 2, 4, 7168, 512, 128),
    # rows too wide, and pairs too many, for one launch
    (3, 2, 4, 8256, 64, 64), (11000, 3, 9, 64, 64, 64), (40000, 1, 17, 192, 130, 2),
    # output rows in the hidden rows' place: fewer and more columns than these
    (37, 2, 4, 256, 2112, 64), (1, 1, 2, 64, 4096, 64), (1500, 3, 5, 1088, 320, 64), (4100, 2, 4, 192, 1088, 64), (600, 4, 3, 512, 512, 128),
    (2049, 8, 16, 640, 384, 128)]


def layers(gen, e, width, hidden, b):
    def one(held, cin, gated):
        return hatq.hatq_pack_linear(torch.randint(-127, 128, (e, held, cin), generator=gen, device=DEV).to(torch.int8),
                                     torch.rand((e, held), generator=gen, device=DEV) / 64 / cin ** 0.5,
                                     torch.randn((e, held), generator=gen, device=DEV) * 0.1, hblock=b, gated=gated)
    return one(2 * hidden, width, True), one(width, hidden, False)


def routing(rng, tokens, topk, e):
    """Some experts more popular, some pairs masked, a token with no expert."""
    p = rng.dirichlet(np.full(e, 0.7))
    ids = rng.choice(e, (tokens, topk), p=p).astype(np.int32)
    ids[rng.random((tokens, topk)) < 0.05] = -1
    if tokens > 2:
        ids[tokens // 2] = (e, -1, 2 ** 31 - 1, -2 ** 31)[:topk] + (e,) * max(0, topk - 4)
    return dev(ids), dev(rng.uniform(0, 1, (tokens, topk)).astype(np.float32))


def by_steps(w_in, w_out, x, ids, weights, dtype):
    ends, src, pos = hatq.hatq_expert_order(ids, w_in.experts)
    hidden = hatq.hatq_experts_int8(w_in, *hatq.hatq_token_quant(x, w_in.w.hblock), ends, src)
    rows = hatq.hatq_experts_int8(w_out, *hatq.hatq_token_quant(hidden, w_out.w.hblock), ends)
    return hatq.hatq_expert_combine(rows, pos, weights, out_dtype=dtype)


def assert_same_bits(a, b):
    bits = torch.int32 if a.dtype == torch.float32 else torch.int16
    nan = torch.isnan(b)
    assert torch.equal(torch.isnan(a), nan)
    assert torch.equal(a.contiguous().view(bits)[~nan], b.view(bits)[~nan])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,topk,e,width,hidden,b", BLOCKS)
def test_block_is_its_steps(dtype, tokens, topk, e, width, hidden, b):
    rng = np.random.default_rng(tokens + width)
    gen = torch.Generator(device=DEV).manual_seed(tokens + hidden)
    w_in, w_out = layers(gen, e, width, hidden, b)
    x = torch.randn((tokens, width + 3), generator=gen, device=DEV).to(dtype)[:, 1:1 + width]
    if tokens > 4:
        x[tokens - 1, 3] = float("inf")                # a token without codes: only its outputs are NaN
    ids, weights = routing(rng, tokens, topk, e)
    if tokens > 4:
        ids[tokens - 1, 0] = 0
    ws = Guarded((hatq.hatq_expert_mlp_ws_bytes(w_in, w_out, tokens, topk),), torch.int8)
    y = Guarded((tokens, width), dtype)
    hatq.hatq_expert_mlp(w_in, w_out, x, ids, weights, y=y.view, ws=ws.view)
    ws.check("workspace")
    y.check()
    ref = by_steps(w_in, w_out, x, ids, weights, dtype)
    assert_same_bits(y.view, ref)
    if tokens > 4:
        assert bool(torch.isnan(ref[tokens - 1]).all()) and not bool(torch.isnan(ref[:tokens - 1]).any())
        assert not bool(ref[tokens // 2].any())        # every pair masked


@pytest.mark.parametrize("tokens,topk,e,width,hidden,b", [(203, 4, 7, 2048, 128, 128), (600, 4, 3, 512, 512, 128), (11000, 3, 9, 64, 64, 64)])
def test_block_in_a_graph_and_on_a_stream(tokens, topk, e, width, hidden, b):
    """Replayed with other tokens and routings in the same buffers, between eager calls."""
    rng = np.random.default_rng(tokens)
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    w_in, w_out = layers(gen, e, width, hidden, b)
    mlp = experts.ExpertMLP(w_in, w_out)
    x = torch.randn((tokens, width), generator=gen, device=DEV).bfloat16()
    ids, weights = routing(rng, tokens, topk, e)
    want = mlp(x, ids, weights)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mlp(x, ids, weights, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    y = torch.empty_like(want)
    ws = torch.empty(hatq.hatq_expert_mlp_ws_bytes(w_in, w_out, tokens, topk), dtype=torch.int8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hatq.hatq_expert_mlp(w_in, w_out, x, ids, weights, y=y, ws=ws)
    for k in range(4):
        x.copy_(torch.randn((tokens, width), generator=gen, device=DEV))
        new = routing(rng, tokens, topk, e)
        ids.copy_(new[0])
        weights.copy_(new[1])
        want = by_steps(w_in, w_out, x, ids, weights, torch.bfloat16)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), k
