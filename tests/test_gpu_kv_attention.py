"""Attention over the INT8 cache against the definition in 64 bits.

Tolerance, per output value, with p the softmax weights and v the values of the 64-bit reference:
rounding of a weight to binary16 2^-11 p |v| (below its normal range 2^-25 of the largest weight's
unit a token, i.e. n 2^-25 max|v|); FP32 scores 2^-20 of c sum|q k|, twice (numerator and
denominator); q held to max|q| / (127 * 508) a value, c max|q| sum|k| 1.6e-5 a score, twice;
binary16 result 2^-11 (2^-25)."""
import math

import numpy as np
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_cache import dev, make_table, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def setup(lens, news, q_heads, kv_heads, dim, page, seed=0, spread=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    table, pages = make_table([max(n, 0) for n in lens], page, seed=seed)
    cache = list(binding.kv_cache_s8(pages, kv_heads, page, dim))
    for i in range(2):
        cache[i] = (torch.randn(pages, kv_heads, page, dim, generator=g, device="cuda") * 40).round().clamp(-127, 127).to(torch.int8)
        cache[2 + i] = 0.02 * torch.exp(spread * torch.randn(pages, kv_heads, generator=g, device="cuda"))
    q = torch.randn(sum(news), q_heads, dim, generator=g, device="cuda").half()
    return tuple(cache), table, q


def reference(q, cache, table, lens, news, window, scale):
    k, v, ks, vs = cache
    heads, page, dim = k.shape[1:]
    out, tol, at = [], [], 0
    for b, (L, n) in enumerate(zip(lens, news)):
        x = q[at:at + n].double().view(n, heads, q.shape[1] // heads, dim)
        at += n
        if L == 0:
            out.append(torch.zeros(n, q.shape[1], dim, dtype=torch.float64, device="cuda"))
            tol.append(torch.zeros_like(out[-1]))
            continue
        slots = dev(table[b, :-(-L // page)]).long()
        kk, vv = ((c[slots].double() * s[slots].double()[..., None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, :L]
                  for c, s in ((k, ks), (v, vs)))
        sc = torch.einsum("nhgd,htd->nhgt", x, kk) * scale
        mag = torch.einsum("nhgd,htd->nhgt", x.abs(), kk.abs()) * scale
        held = x.abs().amax(3, keepdim=True) * kk.abs().sum(2).amax(1)[None, :, None, None] * (scale / (127 * 508))
        pos = L - n + torch.arange(n, device="cuda")[:, None]
        tok = torch.arange(L, device="cuda")[None]
        hidden = tok > pos
        if window:
            hidden = hidden | (tok <= pos - window)
        sc = sc.masked_fill(hidden[:, None, None, :], -math.inf)
        w = torch.nan_to_num(torch.softmax(sc, dim=3), nan=0.0)       # rows that see nothing
        o = torch.einsum("nhgt,htd->nhgd", w, vv)
        mass = torch.einsum("nhgt,htd->nhgd", w, vv.abs())
        rel = 2.0 ** -11 + 2 * 2.0 ** -20 * mag.amax(3, keepdim=True) + 2 * held + 4e-6
        t = rel * mass + 2.0 ** -11 * o.abs() + 2.0 ** -25 * (1 + L * vv.abs().amax())
        out.append(o.reshape(n, q.shape[1], dim))
        tol.append(t.reshape(n, q.shape[1], dim))
    return torch.cat(out), torch.cat(tol)


def check(lens, news, q_heads, kv_heads, dim, page, window=0, seed=0, spread=1.0, strided=False):
    cache, table, q = setup(lens, news, q_heads, kv_heads, dim, page, seed, spread)
    scale = dim ** -0.5
    if strided:                        # as one projection leaves them, and heads in front of tokens
        wide = torch.zeros(q.shape[0], q_heads + 2 * kv_heads, dim, device="cuda", dtype=torch.float16)
        wide[:, :q_heads] = q
        q = wide[:, :q_heads]
    cu = dev(starts(news))
    got = binding.kv_attention_s8(q, cache, cu, dev(lens), dev(table), max(news + [1]), window=window)
    ref, tol = reference(q, cache, table, lens, news, window, scale)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol.clamp(min=1e-30)).max().item()
    again = binding.kv_attention_s8(q, cache, cu, dev(lens), dev(table), max(news + [1]), window=window)
    assert torch.equal(got, again)     # splits are joined in a fixed order
    return got


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_single_tokens(dim, page):
    check([1, 15, 16, 17, 127, 128, 129, 500, 1023], [1] * 9, 8, 2, dim, page)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (4, 4), (6, 2), (32, 8), (12, 1), (16, 1), (40, 2), (64, 1)])
def test_head_layouts(q_heads, kv_heads):
    for dim in (64, 128, 256):
        check([300, 77], [1, 1], q_heads, kv_heads, dim, 32)
        check([300, 77, 5], [3, 1, 4], q_heads, kv_heads, dim, 16, seed=1)


@pytest.mark.parametrize("lens,news", [
    ([0, 5, 0, 40], [1, 1, 0, 2]),            # empty sequences, with and without a query
    ([3, 1, 2], [5, 4, 2]),                   # queries in front of the first token see nothing
    ([1], [1]), ([131], [131]), ([1000], [64]), ([700, 90, 2000], [650, 90, 1]),
    ([16, 32, 48], [16, 17, 33]), ([0], [3])])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_lengths(lens, news, dim):
    check(lens, news, 8, 2, dim, 16)
    check(lens, news, 3, 3, dim, 64, seed=2, strided=True)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 5000])
def test_windows(window):
    check([1, 16, 333, 1000], [1, 1, 1, 1], 8, 2, 128, 16, window=window)
    check([40, 333, 1000], [33, 64, 200], 4, 1, 64, 32, window=window, seed=3)


@pytest.mark.parametrize("L", [4096, 20011, 70001])
def test_long_single_sequence(L):
    check([L], [1], 8, 2, 128, 64)
    check([L], [4], 8, 8, 64, 16, seed=4)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,news,q_heads,kv_heads", [
    ([9000], [40], 4, 1), ([5000, 100, 4096], [70, 33, 300], 4, 2), ([20000, 3], [17, 1], 8, 1)])
def test_chunks_over_long_sequences(dim, lens, news, q_heads, kv_heads):
    """Few row tiles: their tokens are divided over CTAs; and a window that leaves most parts nothing."""
    check(lens, news, q_heads, kv_heads, dim, 64, seed=7)
    check(lens, news, q_heads, kv_heads, dim, 16, window=300, seed=8)


def test_chunks_of_many_sequences():
    """Row tiles of sequences of all lengths, longest first, beside sequences of single tokens."""
    g = np.random.default_rng(11)
    news = [int(x) for x in g.integers(0, 130, 45)]
    lens = [n + int(x) for n, x in zip(news, g.integers(0, 1500, 45))]
    news[7], news[20] = 1, 1
    check(lens, news, 4, 1, 64, 16)
    check(lens, news, 4, 4, 128, 32, window=77)


def test_many_sequences():
    g = np.random.default_rng(5)
    lens = [int(x) for x in g.integers(0, 900, 300)]
    news = [min(1, n) if i % 7 else 2 for i, n in enumerate(lens)]
    check(lens, news, 4, 2, 64, 16)


def test_scales_of_very_different_size():
    """The value scale is folded into the weights' exponent: pages may differ by orders of magnitude."""
    check([600, 1200], [1, 2], 8, 2, 128, 16, spread=4.0, seed=6)


def test_one_token_dominates():
    """A score far above the rest: the weights of everything else vanish, also across CTAs' joins."""
    cache, table, q = setup([2000], [1], 4, 1, 128, 16)
    k, v, ks, vs = cache
    slot, at = table[0, 777 // 16], 777 % 16
    ks.fill_(0.05)
    q[0] = 8 * torch.sign(k[slot, 0, at].float()).half()
    got = binding.kv_attention_s8(q, cache, dev([0, 1]), dev([2000]), dev(table), 1)
    want = (v[slot, 0, at].double() * vs[slot, 0].double()).half()
    assert torch.equal(got[0], want.expand(4, -1))


def test_page_of_zeros_and_stale_contents():
    """Tokens of an all-zero page count in the denominator; what lies behind a sequence's end does not, whatever
    the scales of pages nobody asked for are."""
    dim, page = 64, 16
    cache, table, q = setup([40], [1], 2, 1, dim, page)
    k, v, ks, vs = cache
    zero = int(table[0, 1])
    k[zero], v[zero], ks[zero], vs[zero] = 0, 0, 0, 0
    used = [int(x) for x in table[0, :3]]
    for s in range(k.shape[0]):
        if s not in used:
            ks[s] = vs[s] = float("nan")
    got = binding.kv_attention_s8(q, cache, dev([0, 1]), dev([40]), dev(table), 1)
    ref, tol = reference(q, cache, table, [40], [1], 0, dim ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()
    vs[used[2]] = float("nan")
    assert torch.isnan(binding.kv_attention_s8(q, cache, dev([0, 1]), dev([40]), dev(table), 1)).all()
    got = binding.kv_attention_s8(q, cache, dev([0, 1]), dev([32]), dev(table), 1)
    assert torch.isfinite(got).all()


def test_output_pitch_and_stream():
    cache, table, q = setup([90, 33], [2, 1], 8, 2, 128, 16)
    stream = torch.cuda.Stream()
    big = torch.full((3, 8 * 128 + 64), 7.0, device="cuda", dtype=torch.float16)
    out = big[:, :1024].view(3, 8, 128)
    cu, lens, tb = dev([0, 2, 3]), dev([90, 33]), dev(table)
    torch.cuda.synchronize()
    binding.kv_attention_s8(q, cache, cu, lens, tb, 2, out=out, stream=stream)
    stream.synchronize()
    ref, tol = reference(q, cache, table, [90, 33], [2, 1], 0, 128 ** -0.5)
    assert ((out.double() - ref).abs() <= tol).all() and (big[:, 1024:] == 7.0).all()


def test_captured_into_a_graph():
    cache, table, q = setup([900], [1], 8, 2, 128, 16)
    cu, lens, tb = dev([0, 1]), dev([900]), dev(table)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        binding.kv_attention_s8(q, cache, cu, lens, tb, 1, out=out)      # scratch exists before the capture
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.kv_attention_s8(q, cache, cu, lens, tb, 1, out=out)
    want = out.clone()
    lens.fill_(500)                    # lengths are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    ref, tol = reference(q, cache, table, [500], [1], 0, 128 ** -0.5)
    assert ((out.double() - ref).abs() <= tol).all() and not torch.equal(out, want)


def test_bad_indices_are_reported_and_not_followed():
    cache, table, q = setup([64], [1], 4, 1, 64, 16)
    pages = cache[0].shape[0]
    for bad in (pages, -1, 2 ** 31 - 1):
        t = dev(table)
        t[0, 2] = bad
        binding.kv_attention_s8(q, cache, dev([0, 1]), dev([64]), t, 1)
        assert binding.gemm_last_device_status() == 6
    for cu, L, bound in (([0, 1], -5, 1), ([0, 1], 10 ** 9, 1), ([1, 0], 64, 1)):
        t = dev(np.where(table < 0, 0, table))
        binding.kv_attention_s8(q, cache, dev(cu), dev([L]), t, bound)
        assert binding.gemm_last_device_status() == 6


def test_write_then_attend():
    """Cache written token by token, then read by the attention: the chain a decoder runs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    heads, dim, page, n = 2, 128, 16, 50
    table, pages = make_table([n], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    qkv = torch.randn(n, 8 + 2 * heads, dim, generator=g, device="cuda").half()
    tb = dev(table)
    outs = []
    for lo, hi in [(0, 20), (20, 21), (21, 22), (22, 40), (40, 50)]:
        rows, cu = qkv[lo:hi], dev([0, hi - lo])
        binding.kv_append_s8(cache, rows[:, 8:8 + heads], rows[:, 8 + heads:], cu, dev([lo]), tb, hi - lo)
        out = binding.kv_attention_s8(rows[:, :8], cache, cu, dev([hi]), tb, hi - lo)
        ref, tol = reference(rows[:, :8], cache, table, [hi], [hi - lo], 0, dim ** -0.5)
        assert ((out.double() - ref).abs() <= tol).all()
        outs.append(out)
    # and against attention over the unquantised keys and values: 8-bit codes are off by half a step each
    k, v = qkv[:, 8:8 + heads].double(), qkv[:, 8 + heads:].double()
    sc = torch.einsum("nhgd,thd->nhgt", qkv[:, :8].double().view(n, heads, -1, dim), k) * dim ** -0.5
    sc = sc.masked_fill(torch.triu(torch.ones(n, n, device="cuda", dtype=torch.bool), 1)[:, None, None], -math.inf)
    full = torch.einsum("nhgt,thd->nhgd", sc.softmax(3), v).reshape(n, 8, dim)
    assert (torch.cat(outs).double() - full).norm() / full.norm() < 0.05
