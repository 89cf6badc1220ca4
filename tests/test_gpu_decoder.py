"""The halves of a decoder layer: a prompt, steps and a mixed batch through them are the calls
they are made of, bit for bit, with INT8 and with 4-bit layers, and the attention in them is
that of the cached values in 64 bits; captured and replayed as a graph over growing
sequences."""
import numpy as np
import pytest
import torch

from cache4_util import attention64, check, held, most_scale
from gpu_util import DEV, dev, host
from paper_2608_01653_amd import decoder, hatq

pytestmark = pytest.mark.gpu
WIDTH, Q_HEADS, HEADS, DIM, HBLOCK, PAGE = 256, 8, 2, 64, 64, 16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    hatq.load()
    torch.cuda.init()


def layer(rng, cout, cin, kind, gated=False):
    w = torch.from_numpy((rng.normal(size=(cout * (2 if gated else 1), cin)) / np.sqrt(cin)).astype(np.float32)).to(DEV)
    if kind == "int8":
        return hatq.hatq_prepare_linear(w, hblock=64, gated=gated)
    return hatq.hatq_prepare_linear4(w, hblock=64, group=64, gated=gated)


def block(rng, kind, pages=64):
    cache = hatq.hatq_cache4_init(pages, PAGE, HEADS, DIM, hblock=HBLOCK, device=DEV)
    cache.buf.fill_(-1)
    return decoder.CachedAttention(layer(rng, (Q_HEADS + 2 * HEADS) * DIM, WIDTH, kind), layer(rng, WIDTH, Q_HEADS * DIM, kind), cache, Q_HEADS)


def tokens(rng, rows, dtype=torch.bfloat16):
    return torch.from_numpy(rng.normal(size=(rows, WIDTH)).astype(np.float32)).to(dtype).to(DEV)


@pytest.mark.parametrize("kind", ["int8", "int4"])
def test_a_prompt_steps_and_a_mixed_batch(kind):
    rng = np.random.default_rng(1)
    att = block(rng, kind)
    table = dev(rng.permutation(64)[:24].reshape(3, 8).astype(np.int32))
    seen = [[], [], []]         # each sequence's keys and values, as the cache got them
    lens = np.zeros(3, np.int32)
    # a prompt of the first two, a step, then a prompt of the third beside steps of the others
    for new in ([70, 33, 0], [1, 1, 0], [1, 1, 41], [1, 4, 1]):
        x = tokens(rng, sum(new))
        lens += np.array(new, np.int32)
        ends = dev(np.cumsum(new).astype(np.int32))
        got = att(x, table, dev(lens), ends)
        qkv = decoder.forward(att.w_qkv, x)
        q, k, v = (t.unflatten(1, (-1, DIM)) for t in qkv.split((Q_HEADS * DIM, HEADS * DIM, HEADS * DIM), dim=1))
        y = hatq.hatq_attention4(att.cache, q, table, dev(lens), ends)
        assert torch.equal(got, decoder.forward(att.w_out, y.reshape(sum(new), -1)))
        row = 0
        for i, n in enumerate(new):
            seen[i].append((k[row:row + n].float().cpu().numpy(), v[row:row + n].float().cpu().numpy()))
            kk, vv = (np.concatenate([s[j] for s in seen[i]]) for j in (0, 1))
            y64, bound = attention64(q[row:row + n].float().cpu().numpy(), held(kk, HBLOCK), held(vv, HBLOCK), most_scale(vv, HBLOCK), HBLOCK,
                                     DIM ** -0.5, True, 0, False)
            check(y[row:row + n].cpu(), y64, bound, f"sequence {i}, {n} rows")
            row += n


def test_rotated_queries_and_keys():
    rng = np.random.default_rng(2)
    att = block(rng, "int4")
    table, lens = dev(np.arange(4, dtype=np.int32).reshape(1, 4)), dev(np.array([20], np.int32))
    x = tokens(rng, 20, torch.float32)
    got = att(x, table, lens, rotate=lambda q, k: (q.flip(0), -k))
    q, k, v = decoder.forward(att.w_qkv, x).unflatten(1, (-1, DIM)).split((Q_HEADS, HEADS, HEADS), dim=1)
    kk, vv = (t.cpu().numpy() for t in (-k, v))
    y64, bound = attention64(q.flip(0).cpu().numpy(), held(kk, HBLOCK), held(vv, HBLOCK), most_scale(vv, HBLOCK), HBLOCK, DIM ** -0.5, True, 0, True)
    y = hatq.hatq_attention4(att.cache, q.flip(0), table, lens)
    check(y, y64, bound, "rotated")
    assert torch.equal(got, decoder.forward(att.w_out, y.reshape(20, -1)))


@pytest.mark.parametrize("kind", ["int8", "int4"])
def test_gated_mlp(kind):
    rng = np.random.default_rng(3)
    mlp = decoder.GatedMLP(layer(rng, 320, WIDTH, kind, gated=True), layer(rng, WIDTH, 320, kind))
    for rows in (1, 30):
        x = tokens(rng, rows)
        assert torch.equal(mlp(x), decoder.forward(mlp.w_out, decoder.forward(mlp.w_in, x)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = mlp(x, stream=side)
    side.synchronize()
    assert torch.equal(y, mlp(x))


def test_a_layer_captured_and_replayed():
    """A whole step of attention and feed-forward as one graph over growing sequences, beside
    eager steps of another cache on the same inputs."""
    rng = np.random.default_rng(4)
    one = block(rng, "int4")
    two = decoder.CachedAttention(one.w_qkv, one.w_out, hatq.hatq_cache4_init(64, PAGE, HEADS, DIM, hblock=HBLOCK, device=DEV), Q_HEADS)
    mlp = decoder.GatedMLP(layer(rng, 320, WIDTH, "int4", gated=True), layer(rng, WIDTH, 320, "int4"))
    table = dev(rng.permutation(64)[:16].reshape(2, 8).astype(np.int32))
    lens = dev(np.array([40, 12], np.int32))
    prompt, ends = tokens(rng, 52), dev(np.array([40, 52], np.int32))
    for att in (one, two):
        att(prompt, table, lens, ends)
    x = tokens(rng, 2)

    def step(att):
        h = x + att(x, table, lens)
        return h + mlp(h)

    lens += 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(one)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step(one)
    lens -= 1
    for _ in range(5):
        lens += 1
        x.copy_(tokens(rng, 2))
        graph.replay()
        eager = step(two)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_refusals():
    rng = np.random.default_rng(5)
    cache = hatq.hatq_cache4_init(4, PAGE, HEADS, DIM, device=DEV)
    qkv, out = layer(rng, (Q_HEADS + 2 * HEADS) * DIM, WIDTH, "int4"), layer(rng, WIDTH, Q_HEADS * DIM, "int4")
    decoder.CachedAttention(qkv, out, cache, Q_HEADS)
    for bad in ((out, out, cache, Q_HEADS), (qkv, qkv, cache, Q_HEADS), (qkv, out, cache, 7), (layer(rng, 384, WIDTH, "int4", gated=True), out, cache, Q_HEADS)):
        with pytest.raises(ValueError):
            decoder.CachedAttention(*bad)
    for bad in ((qkv, out), (layer(rng, 100, 128, "int8", gated=True), out)):
        with pytest.raises(ValueError):
            decoder.GatedMLP(*bad)
