"""Attention of prompts over their own binary16 keys and values against the definition in 64 bits.

Tolerance, per output value, with p the softmax weights and v the values of the 64-bit reference:
rounding of a weight to binary16 2^-11 p |v| (below its normal range 2^-32 of the largest a token); FP32
scores 2^-20 of c sum|q k|, twice (numerator and denominator); sums cut off 2e-9 a token; binary16
result 2^-11 (2^-25)."""
import math

import numpy as np
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def reference(q, k, v, lens, causal, window, scale):
    outs, tols, at = [], [], 0
    heads = k.shape[1]
    for n in lens:
        x = q[at:at + n].double().view(n, heads, q.shape[1] // heads, q.shape[2])
        kk, vv = k[at:at + n].double(), v[at:at + n].double()
        at += n
        pos, tok = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        hidden = (tok > pos) if causal else torch.zeros(n, n, dtype=torch.bool, device="cuda")
        if window:
            hidden = hidden | (tok <= pos - window)
        for lo in range(0, n, 512):
            sl = slice(lo, lo + 512)
            sc = torch.einsum("nhgd,thd->nhgt", x[sl], kk) * scale
            mag = torch.einsum("nhgd,thd->nhgt", x[sl].abs(), kk.abs()).amax(3, keepdim=True) * scale
            w = torch.softmax(sc.masked_fill(hidden[sl][:, None, None], -math.inf), dim=3)
            o = torch.einsum("nhgt,thd->nhgd", w, vv)
            mass = torch.einsum("nhgt,thd->nhgd", w, vv.abs())
            t = (2.0 ** -11 + 2 * 2.0 ** -20 * mag + 4e-6 + 2e-9 * n) * mass + 2.0 ** -11 * o.abs()
            t = t + 2.0 ** -25 + n * 2.0 ** -32 * vv.abs().amax()
            outs.append(o.reshape(-1, *q.shape[1:]))
            tols.append(t.reshape(-1, *q.shape[1:]))
    return torch.cat(outs), torch.cat(tols)


def make(tokens, q_heads, kv_heads, dim, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows = torch.randn(tokens, q_heads + 2 * kv_heads, dim, generator=g, device="cuda").half()
    return rows[:, :q_heads], rows[:, q_heads:q_heads + kv_heads], rows[:, q_heads + kv_heads:]


def check(lens, q_heads, kv_heads, dim, causal=True, window=0, seed=0, scale=None):
    q, k, v = make(sum(lens), q_heads, kv_heads, dim, seed)
    cu = dev(starts(lens))
    got = binding.attention_fp16(q, k, v, cu, max(lens), softmax_scale=scale, causal=causal, window=window)
    ref, tol = reference(q, k, v, lens, causal, window, dim ** -0.5 if scale is None else scale)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol).max().item()
    again = binding.attention_fp16(q, k, v, cu, max(lens), softmax_scale=scale, causal=causal, window=window)
    assert torch.equal(got, again)
    return got


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700])
def test_lengths(n, dim):
    check([n], 8, 2, dim)
    check([n], 2, 2, dim, causal=False, seed=1)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (4, 4), (6, 2), (32, 8), (12, 1), (24, 8), (40, 2), (64, 1), (128, 1), (100, 1)])
def test_head_layouts(q_heads, kv_heads):
    for dim in (64, 128, 256):
        check([130, 77], q_heads, kv_heads, dim)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens", [[0, 5, 0, 40], [1, 1, 1], [300, 0, 1, 512, 77], [128, 256, 128, 1]])
def test_packed(lens, dim):
    check(lens, 8, 2, dim)
    check(lens, 3, 3, dim, causal=False, seed=2)


def test_many_sequences():
    """Row tiles of sequences of all lengths, longest first, several per CTA."""
    g = np.random.default_rng(11)
    lens = [int(x) for x in g.integers(0, 400, 90)]
    check(lens, 8, 2, 128)
    check(lens, 4, 4, 64, window=50, seed=1)
    check(lens, 4, 1, 256, causal=False, seed=2)


@pytest.mark.parametrize("window", [1, 2, 127, 128, 129, 1000, 100000])
def test_windows(window):
    check([40, 333, 1000], 8, 2, 128, window=window)
    check([1500], 4, 4, 64, window=window, seed=1)
    check([700], 4, 1, 256, window=window, seed=2)


@pytest.mark.parametrize("n,dim", [(5000, 128), (9001, 64), (3001, 256)])
def test_long(n, dim):
    check([n], 8, 2, dim)


def test_scores_of_every_size():
    """Scales that make the softmax flat, and so steep that a row is one token: its maximum moves often."""
    for scale in (1e-4, 1.0, 8.0):
        check([900, 200], 4, 2, 128, scale=scale, seed=3)


def test_rising_scores():
    """Every tile of tokens has a larger maximum than the one before."""
    q, k, v = (t.contiguous() for t in make(1024, 2, 1, 128, seed=4))
    q.fill_(1.0)
    k.copy_((torch.arange(1024, device="cuda") / 64.0)[:, None, None].expand_as(k))
    got = binding.attention_fp16(q, k, v, dev([0, 1024]), 1024)
    ref, tol = reference(q, k, v, [1024], True, 0, 128 ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_hidden_values_that_are_not_finite(dim, bad):
    """Tokens behind a query, in front of its window and of the next sequence leave it alone, whatever they hold."""
    lens = [300, 90]
    for window in (0, 40):
        q, k, v = (t.contiguous() for t in make(sum(lens), 4, 2, dim, seed=5))
        clean = binding.attention_fp16(q, k, v, dev(starts(lens)), 300, window=window)
        for t, name in ((200, "v"), (200, "k"), (300, "v"), (299, "v")):
            kk, vv = k.clone(), v.clone()
            (vv if name == "v" else kk)[t, 1, 3] = bad
            got = binding.attention_fp16(q, kk, vv, dev(starts(lens)), 300, window=window)
            end = 300 if t < 300 else 390
            sees = torch.zeros(390, 4, dtype=torch.bool, device="cuda")
            sees[t:min(end, t + window) if window else end, 2:] = True
            # (rows computed alone have their sums in another order)
            near = (got.float() - clean.float()).abs() <= 2.0 ** -9 * clean.float().abs().amax()
            assert near[~sees].all()
            if name == "v":
                assert (~torch.isfinite(got[..., 3]))[sees].all() and near[..., :3][sees].all() and near[..., 4:][sees].all()
            elif bad != bad:
                assert torch.isnan(got[sees]).all()


def test_queries_that_are_not_finite():
    q, k, v = (t.contiguous() for t in make(150, 4, 2, 128, seed=6))
    clean = binding.attention_fp16(q, k, v, dev([0, 150]), 150)
    q[70, 1, 5], q[0, 0, 0] = float("inf"), float("nan")
    got = binding.attention_fp16(q, k, v, dev([0, 150]), 150)
    bad = torch.zeros(150, 4, dtype=torch.bool, device="cuda")
    bad[70, 1] = bad[0, 0] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])


def test_layouts_of_the_operands():
    """Heads in front of tokens, odd pitches, an output with a pitch of its own; rows behind the last sequence stay."""
    lens = [100, 33]
    q, k, v = (t.contiguous() for t in make(140, 6, 2, 64, seed=7))
    want = binding.attention_fp16(q, k, v, dev(starts(lens)), 100)[:133]
    ht = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    out = torch.full((140, 6 * 64 + 24), 7.0, device="cuda", dtype=torch.float16)
    view = out[:, :384].view(140, 6, 64)
    binding.attention_fp16(*ht, dev(starts(lens)), 100, out=view)
    assert torch.equal(view[:133], want) and (out[:, 384:] == 7).all() and (out[133:] == 7).all()
    pitched = [torch.zeros(140, t.shape[1], 72, device="cuda", dtype=torch.float16)[..., :64].copy_(t) for t in (q, k, v)]
    odd = [torch.zeros(140, t.shape[1] * 64 + 40, device="cuda", dtype=torch.float16)[:, 8:8 + t.shape[1] * 64].view(140, -1, 64).copy_(t)
           for t in (q, k, v)]
    assert torch.equal(binding.attention_fp16(*pitched, dev(starts(lens)), 100)[:133], want)
    assert torch.equal(binding.attention_fp16(*odd, dev(starts(lens)), 100)[:133], want)


def test_stream_and_graph():
    q, k, v = (t.contiguous() for t in make(400, 8, 2, 128, seed=8))
    cu = dev([0, 250, 400])
    want = binding.attention_fp16(q, k, v, cu, 400)
    side, out = torch.cuda.Stream(), torch.empty_like(q)
    torch.cuda.synchronize()
    got = binding.attention_fp16(q, k, v, cu, 400, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.attention_fp16(q, k, v, cu, 400, out=out)
    cu.copy_(dev([0, 100, 400]))        # lengths are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, binding.attention_fp16(q, k, v, cu, 400)) and not torch.equal(out, want)


def test_bad_counts_are_reported_and_not_followed():
    q, k, v = (t.contiguous() for t in make(64, 4, 2, 64, seed=9))
    want = binding.attention_fp16(q, k, v, dev([0, 64]), 64)
    for cu, most in (([0, 70], 100), ([-3, 20], 64), ([30, 10], 64), ([0, 64], 40)):
        got = binding.attention_fp16(q, k, v, dev(cu), most)
        assert binding.gemm_last_device_status() == 6, cu
        if cu == [0, 64]:
            assert torch.equal(got[:40], want[:40])


def test_refusals():
    q, k, v = make(8, 4, 2, 64)
    cu = dev([0, 8])
    for a in ((q.float(), k, v), (q, k[:4], v), (q, k, v.contiguous()), (q, k[..., :32], v[..., :32]), (q[0], k, v), (q[:4], k, v)):
        with pytest.raises((TypeError, ValueError)):
            binding.attention_fp16(*a, cu, 8)
    for kw in (dict(window=3, causal=False), dict(window=-1), dict(softmax_scale=0.0)):
        with pytest.raises(binding.GemmError):
            binding.attention_fp16(q, k, v, cu, 8, **kw)
    with pytest.raises(binding.GemmError):
        binding.attention_fp16(q[:, :3], k, v, cu, 8)
    with pytest.raises(ValueError):
        binding.attention_fp16(q, k, v, cu, 8, out=torch.empty(8, 4, 32, device="cuda", dtype=torch.float16))
