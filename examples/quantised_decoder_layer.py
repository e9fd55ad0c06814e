"""One transformer decoder layer with INT8 weights, INT8 activations and an INT8 key/value cache, as a
serving program runs it: a ragged batch of prompts first, then token after token.

    python examples/quantised_decoder_layer.py

Per call: rows are normalised (plain torch), quantised, projected (INT8, bias) to queries, keys and values,
the keys and values go to the cache, attention reads the cache, and the two projections back add onto the
residual stream inside their epilogues.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_10103_b200 import binding  # noqa: E402


def quantise_weight(w: torch.Tensor):
    """Rows of a weight matrix (out, in) as int8 codes and scales."""
    return binding.gemm_quantize_rows(w.contiguous(), "s8")


def normalise(x: torch.Tensor) -> torch.Tensor:
    x32 = x.float()
    return (x32 * torch.rsqrt(x32.square().mean(1, keepdim=True) + 1e-6)).half()


class DecoderLayer:
    """width = heads * dim; a two-matrix feed-forward block of `inner` columns with GELU."""

    def __init__(self, heads: int, kv_heads: int, dim: int, inner: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.width = heads, kv_heads, dim, heads * dim

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) / cols ** 0.5).half()

        self.float_weights = dict(qkv=weight((heads + 2 * kv_heads) * dim, self.width), out=weight(self.width, self.width),
                                  up=weight(inner, self.width), down=weight(self.width, inner))
        self.qkv_bias = torch.randn((heads + 2 * kv_heads) * dim, generator=g, device=device) * 0.1
        self.weights = {name: quantise_weight(w) for name, w in self.float_weights.items()}

    def _linear(self, name, x, **kw):
        q, scale = binding.gemm_quantize_rows(x, "s8")
        w, col_scale = self.weights[name]
        return binding.gemm_s8_linear(q, w, scale, col_scale, **kw)

    def forward(self, x, cache, table, cu, past, kv_len, max_new):
        """x: float16 (tokens, width), the new tokens of all sequences; updated in place."""
        h, k, d = self.heads, self.kv_heads, self.dim
        qkv = self._linear("qkv", normalise(x), bias=self.qkv_bias).view(-1, h + 2 * k, d)
        binding.kv_append_s8(cache, qkv[:, h:h + k], qkv[:, h + k:], cu, past, table, max_new)
        a = binding.kv_attention_s8(qkv[:, :h], cache, cu, kv_len, table, max_new)
        self._linear("out", a.view(-1, self.width), residual=x, C=x)
        f = self._linear("up", normalise(x), activation="gelu_tanh")
        return self._linear("down", f, residual=x, C=x)


class Batch:
    """Pages, lengths and the block table of a few sequences."""

    def __init__(self, layer: DecoderLayer, sequences: int, most: int, page: int = 64, device="cuda"):
        per = -(-most // page)
        self.cache = binding.kv_cache_s8(sequences * per, layer.kv_heads, page, layer.dim, device)
        self.table = torch.randperm(sequences * per, device=device).to(torch.int32).view(sequences, per)
        self.length = [0] * sequences
        self.device = device

    def step(self, layer, x, new):
        """Runs the layer on new[b] more tokens of each sequence."""
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        total = [a + n for a, n in zip(self.length, new)]

        def ints(v):
            return torch.tensor(v, dtype=torch.int32, device=self.device)

        y = layer.forward(x, self.cache, self.table, ints(starts), ints(self.length), ints(total), max(new))
        self.length = total
        return y


def main():
    torch.manual_seed(0)
    layer = DecoderLayer(heads=16, kv_heads=4, dim=128, inner=8192)
    prompts = [300, 17, 1024, 1]
    batch = Batch(layer, len(prompts), most=2048)
    y = batch.step(layer, torch.randn(sum(prompts), layer.width, device="cuda").half(), prompts)
    print("prompts of %s tokens: output %s, rms %.3f" % (prompts, tuple(y.shape), y.float().square().mean().sqrt()))
    for _ in range(3):      # the shapes of single tokens run for the first time
        batch.step(layer, torch.randn(len(prompts), layer.width, device="cuda").half(), [1] * len(prompts))
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    x = torch.randn(len(prompts), layer.width, device="cuda").half()
    a.record()
    for _ in range(50):
        batch.step(layer, x, [1] * len(prompts))
    b.record()
    torch.cuda.synchronize()
    print("one token of each: %.1f us a layer" % (a.elapsed_time(b) / 50 * 1e3))
    if binding.gemm_last_device_status() != 0:
        raise SystemExit("a kernel reported an error")


if __name__ == "__main__":
    main()
