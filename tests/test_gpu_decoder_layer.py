"""The example's decoder layer: what a token gets must not depend on how the sequence was cut into calls
beyond the 8-bit roundings, and must follow the same layer in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decoder_example", os.path.join(ROOT, "examples", "quantised_decoder_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def in_64_bits(layer, x):
    h, k, d = layer.heads, layer.kv_heads, layer.dim
    w = {n: v.double() for n, v in layer.float_weights.items()}
    x = x.double()

    def norm(v):
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6)

    qkv = (norm(x) @ w["qkv"].t() + layer.qkv_bias.double()).view(-1, h + 2 * k, d)
    n = x.shape[0]
    sc = torch.einsum("nhgd,thd->nhgt", qkv[:, :h].view(n, k, h // k, d), qkv[:, h:h + k]) / math.sqrt(d)
    sc = sc.masked_fill(torch.triu(torch.ones(n, n, device="cuda", dtype=torch.bool), 1)[:, None, None], -math.inf)
    a = torch.einsum("nhgt,thd->nhgd", sc.softmax(3), qkv[:, h + k:]).reshape(n, -1)
    x = x + a @ w["out"].t()
    f = norm(x) @ w["up"].t()
    f = 0.5 * f * (1 + torch.tanh(math.sqrt(2 / math.pi) * (f + 0.044715 * f ** 3)))
    return x + f @ w["down"].t()


def test_layer_follows_the_definition():
    m = example()
    layer = m.DecoderLayer(heads=8, kv_heads=2, dim=64, inner=1536, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    xs = [torch.randn(n, layer.width, generator=g, device="cuda").half() for n in (70, 5, 130)]
    want = [in_64_bits(layer, x) for x in xs]
    cuts = [[70, 5, 100], [0, 0, 1], [0, 0, 29]], [[40, 1, 0], [30, 1, 64], [0, 1, 33], [0, 1, 1], [0, 1, 32]]
    for cut in cuts:
        batch = m.Batch(layer, 3, most=256, page=16)
        got = [[], [], []]
        for new in cut:
            done = batch.length
            x = torch.cat([v[a:a + n] for v, a, n in zip(xs, done, new)])
            y = batch.step(layer, x, new)
            for b, part in enumerate(y.split(new)):
                got[b].append(part)
        for v, w in zip(got, want):
            v = torch.cat(v).double()
            # roundings to 8 bits: weights, activations (four times) and the cache, each about 1 % of its operand
            assert (v - w).norm() / w.norm() < 0.05


def test_example_runs(capsys):
    example().main()
    assert "us a layer" in capsys.readouterr().out
