"""The example's decoder layer with rotary positions and the cache in 4 bits: the operators around attention one after the
other, against the same layer in 64 bits, whichever way a sequence is cut into calls.

Tolerance, of the output's norm: 0.05 for the roundings to 8 bits (weights and activations, as for the 8-bit cache); and
for keys and values in 4 bits a quarter of the attention's part in the residual stream (each off by 0.1 of a value's size in the
mean of squares, in scores and in the sum; bounded as in the cache's own test), once as it is and once through the feed-forward
block, whose input is normalised, so that a relative change leaves it as about the same one."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_decoder_layer import example

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def in_64_bits(layer, x):
    """The layer's output for one sequence, and the attention's part of it."""
    h, k, d = layer.heads, layer.kv_heads, layer.dim
    w = {n: v.double() for n, v in layer.float_weights.items()}
    x, n = x.double(), x.shape[0]

    def norm(v):
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6)

    qkv = (norm(x) @ w["qkv"].t() + layer.qkv_bias.double()).view(-1, h + 2 * k, d)
    angle = torch.arange(n, device="cuda").double()[:, None] * layer.inv_freq.double()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = qkv[:, :h + k, :d // 2], qkv[:, :h + k, d // 2:]
    turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
    sc = torch.einsum("nhgd,thd->nhgt", turned[:, :h].reshape(n, k, h // k, d), turned[:, h:]) / math.sqrt(d)
    sc = sc.masked_fill(torch.triu(torch.ones(n, n, device="cuda", dtype=torch.bool), 1)[:, None, None], -math.inf)
    part = torch.einsum("nhgt,thd->nhgd", sc.softmax(3), qkv[:, h + k:]).reshape(n, -1) @ w["out"].t()
    x = x + part
    f = norm(x) @ w["up"].t()
    f = 0.5 * f * (1 + torch.tanh(math.sqrt(2 / math.pi) * (f + 0.044715 * f ** 3)))
    return x + f @ w["down"].t(), part


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 64), (4, 4, 128), (6, 1, 256)])
def test_layer_follows_the_definition(heads, kv_heads, dim):
    m = example()
    layer = m.DecoderLayer(heads=heads, kv_heads=kv_heads, dim=dim, inner=1536, seed=3, rotary_base=10000.0, cache="u4")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    xs = [torch.randn(n, layer.width, generator=g, device="cuda").half() for n in (70, 5, 130)]
    want = [in_64_bits(layer, x) for x in xs]
    cuts = [[70, 5, 130]], [[70, 5, 100], [0, 0, 1], [0, 0, 29]], [[40, 1, 0], [30, 1, 64], [0, 1, 33], [0, 1, 1], [0, 1, 32]]
    for cut in cuts:
        batch = m.Batch(layer, 3, most=256, page=16)
        got = [[], [], []]
        for new in cut:
            done = batch.length
            x = torch.cat([v[a:a + n] for v, a, n in zip(xs, done, new)])
            y = batch.step(layer, x, new)
            for b, part in enumerate(y.split(new)):
                got[b].append(part)
        for v, (w, part) in zip(got, want):
            v = torch.cat(v).double()
            assert (v - w).norm() <= 0.05 * w.norm() + 0.5 * part.norm()


def test_prompts_leave_the_8_bit_roundings_only():
    """A whole prompt attends over its own 16-bit keys and values: the bound of the 8-bit roundings alone."""
    m = example()
    layer = m.DecoderLayer(heads=8, kv_heads=2, dim=128, inner=1024, seed=5, rotary_base=500.0, cache="u4")
    xs = [torch.randn(n, layer.width, device="cuda").half() for n in (257, 1, 64)]
    want = torch.cat([in_64_bits(layer, x)[0] for x in xs])
    y = m.Batch(layer, 3, most=512).step(layer, torch.cat(xs), [257, 1, 64])
    assert (y.double() - want).norm() / want.norm() < 0.05


def test_a_step_captured_into_a_graph():
    """Rotation, cache write, attention and the linear layers of one token per sequence, captured once and replayed as the
    sequences grow: positions, lengths and inputs are read when the graph runs."""
    m = example()
    layer = m.DecoderLayer(heads=8, kv_heads=2, dim=128, inner=1024, seed=6, rotary_base=10000.0, cache="u4")
    batch, plain = m.Batch(layer, 2, most=256), m.Batch(layer, 2, most=256)
    plain.table = batch.table
    x = torch.randn(130, layer.width, device="cuda").half()
    batch.step(layer, x.clone(), [100, 30])
    plain.step(layer, x.clone(), [100, 30])

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    cu, past, total, at = ints([0, 1, 2]), ints([100, 30]), ints([101, 31]), ints([100, 30])
    token, side = torch.zeros(2, layer.width, device="cuda", dtype=torch.float16), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(2):          # scratch exists before the capture
            layer.forward(token, batch.cache, batch.table, cu, past, total, 1, at)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.forward(token, batch.cache, batch.table, cu, past, total, 1, at)
    for step in range(3):
        fresh = torch.randn(2, layer.width, device="cuda").half()
        token.copy_(fresh)
        for t, v in ((past, [100 + step, 30 + step]), (at, [100 + step, 30 + step]), (total, [101 + step, 31 + step])):
            t.copy_(ints(v))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, plain.step(layer, fresh, [1, 1]))
