"""Attention over the 4-bit cache against the definition in 64 bits.

Tolerance, per output value, with p the softmax weights, v the values and c the softmax scale: rounding of a weight to
binary16 2^-11 p |v| -- codes count with their distance from the middle of the range, so |v| stands for up to
max(|v|, |offset| + 15 scale) -- (below its normal range 2^-32 of the largest a token); FP32 scores 2^-20 of c sum |q| (|offset|
+ 15 scale), twice (numerator and denominator); q in 16 bits of fixed point, max|q| / 64516 a value (few rows), or v rounded to
binary16, 2^-11 of p |v| (many rows); sums cut off 2e-9 a token; binary16 result 2^-11 (2^-25)."""
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
    cache = list(binding.kv_cache_u4(pages, kv_heads, page, dim))
    for i in range(2):
        cache[i] = torch.randint(0, 256, cache[i].shape, generator=g, device="cuda", dtype=torch.uint8)
        step = 0.2 * torch.exp(spread * torch.randn(pages, kv_heads, page, generator=g, device="cuda"))
        mid = 7.5 + torch.randn(pages, kv_heads, page, generator=g, device="cuda")
        cache[2 + i] = torch.stack((step, -step * mid), dim=3).clamp(-4000, 4000).half()
    q = torch.randn(sum(news), q_heads, dim, generator=g, device="cuda").half()
    return tuple(cache), table, q


def values(codes, scale):
    """Codes [..., dim / 2] and pairs [..., 2] as 64-bit values, and the most a value of that token could be."""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).double()
    s = scale.double()
    return s[..., 1:] + c * s[..., :1], (s[..., 1:].abs() + 15 * s[..., :1].abs()).expand(c.shape)


def reference(q, cache, table, lens, news, window, scale):
    k, v, ks, vs = cache
    heads, page = k.shape[1:3]
    dim = 2 * k.shape[3]
    out, tol, at = [], [], 0
    for b, (L, n) in enumerate(zip(lens, news)):
        x = q[at:at + n].double().view(n, heads, q.shape[1] // heads, dim)
        at += n
        if L == 0:
            out.append(torch.zeros(n, q.shape[1], dim, dtype=torch.float64, device="cuda"))
            tol.append(torch.zeros_like(out[-1]))
            continue
        slots = dev(table[b, :-(-L // page)]).long()
        (kk, ktop), (vv, vtop) = ([t.transpose(0, 1).reshape(heads, -1, dim)[:, :L] for t in values(c[slots], s[slots])]
                                  for c, s in ((k, ks), (v, vs)))
        held = x.abs().amax(3, keepdim=True) * ktop.sum(2).amax(1)[None, :, None, None] * (scale / 64516)
        for lo in range(0, n, 256):
            xs = x[lo:lo + 256]
            sc = torch.einsum("nhgd,htd->nhgt", xs, kk) * scale
            mag = (torch.einsum("nhgd,htd->nhgt", xs.abs(), ktop) * scale).amax(3, keepdim=True)
            pos = L - n + lo + torch.arange(xs.shape[0], device="cuda")[:, None]
            tok = torch.arange(L, device="cuda")[None]
            hidden = tok > pos
            if window:
                hidden = hidden | (tok <= pos - window)
            w = torch.nan_to_num(torch.softmax(sc.masked_fill(hidden[:, None, None, :], -math.inf), dim=3), nan=0.0)
            o = torch.einsum("nhgt,htd->nhgd", w, vv)
            mass = torch.einsum("nhgt,htd->nhgd", w, vtop)
            rel = 2.0 ** -11 + 2 * 2.0 ** -20 * mag + 2 * held[lo:lo + 256] + 4e-6 + 2e-9 * L
            t = rel * mass + 2.0 ** -11 * torch.einsum("nhgt,htd->nhgd", w, vv.abs()) + 2.0 ** -11 * o.abs()
            t = t + 2.0 ** -25 + L * 2.0 ** -32 * vtop.amax()
            out.append(o.reshape(-1, q.shape[1], dim))
            tol.append(t.reshape(-1, q.shape[1], dim))
    return torch.cat(out), torch.cat(tol)


def check(lens, news, q_heads, kv_heads, dim, page, window=0, seed=0, spread=1.0, strided=False):
    cache, table, q = setup(lens, news, q_heads, kv_heads, dim, page, seed, spread)
    scale = dim ** -0.5
    if strided:                        # as one projection leaves them
        wide = torch.zeros(q.shape[0], q_heads + 2 * kv_heads, dim, device="cuda", dtype=torch.float16)
        wide[:, :q_heads] = q
        q = wide[:, :q_heads]
    cu = dev(starts(news))
    got = binding.kv_attention_u4(q, cache, cu, dev(lens), dev(table), max(news + [1]), window=window)
    ref, tol = reference(q, cache, table, lens, news, window, scale)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol.clamp(min=1e-30)).max().item()
    again = binding.kv_attention_u4(q, cache, cu, dev(lens), dev(table), max(news + [1]), window=window)
    assert torch.equal(got, again)     # splits are joined in a fixed order
    return got


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_single_tokens(dim, page):
    check([1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 500, 1023], [1] * 12, 8, 2, dim, page)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (4, 4), (6, 2), (32, 8), (12, 1), (16, 1), (40, 2), (64, 1), (128, 1)])
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


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257])
def test_row_counts(rows):
    """Queries per sequence around the sizes where the kernels and their tiles change."""
    check([rows + 50, rows, 400 + rows], [rows, rows, rows], 1, 1, 128, 32)
    check([600, 300 + rows], [1, rows], 2, 1, 64, 16, seed=1)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 31, 33, 100, 5000])
def test_windows(window):
    check([1, 16, 333, 1000], [1, 1, 1, 1], 8, 2, 128, 16, window=window)
    check([40, 333, 1000], [33, 64, 200], 4, 1, 64, 32, window=window, seed=3)
    check([900, 333], [3, 1], 4, 1, 256, 128, window=window, seed=4)


@pytest.mark.parametrize("L", [4096, 20011, 70001])
def test_long_single_sequence(L):
    check([L], [1], 8, 2, 128, 64)
    check([L], [4], 8, 8, 64, 16, seed=4)
    check([L], [2], 4, 2, 256, 32, seed=5)


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
    """The value scale is folded into the weights' exponent: tokens may differ by orders of magnitude."""
    check([600, 1200], [1, 2], 8, 2, 128, 16, spread=2.0, seed=6)


def test_one_token_dominates():
    """A score far above the rest: the weights of everything else vanish, also across CTAs' joins."""
    cache, table, q = setup([2000], [1], 4, 1, 128, 16)
    k, v, ks, vs = cache
    slot, at = int(table[0, 777 // 16]), 777 % 16
    ks[..., 0], ks[..., 1] = 0.5, -3.75
    kk, _ = values(k[slot, 0, at], ks[slot, 0, at])
    q[0] = 8 * torch.sign(kk).half()
    got = binding.kv_attention_u4(q, cache, dev([0, 1]), dev([2000]), dev(table), 1)
    want = values(v[slot, 0, at], vs[slot, 0, at])[0]
    assert ((got[0].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -20 * want.abs().amax()).all()


@pytest.mark.parametrize("news", [1, 3, 40])
def test_tokens_that_are_not_finite(news):
    """NaN for the queries that see them; hidden ones, and pages nobody asked for, leave a result alone."""
    dim, page, L = 128, 16, 90
    for window in (0, 20):
        cache, table, q = setup([L, 50], [news, 1], 4, 2, dim, page, seed=3)
        args = (dev(starts([news, 1])), dev([L, 50]), dev(table), news)
        clean = binding.kv_attention_u4(q, cache, *args, window=window)
        used = [int(x) for x in table.ravel() if x >= 0]
        for s in range(cache[0].shape[0]):
            if s not in used:
                cache[2][s] = cache[3][s] = float("nan")
        for which in (2, 3):
            for part in (0, 1):
                for t in (0, 60, 88, 89, 91, 95):
                    bad = [x.clone() for x in cache]
                    slot = int(table[0, t // page])
                    bad[which][slot, 1, t % page, part] = float("inf") if t % 2 else float("nan")
                    got = binding.kv_attention_u4(q, tuple(bad), *args, window=window)
                    pos = L - news + torch.arange(news, device="cuda")
                    sees = (pos >= t) & (t < L)
                    if window:
                        sees &= t > pos - window
                    nan = torch.zeros(news + 1, 4, dtype=torch.bool, device="cuda")
                    nan[:news, 2:] = sees[:, None]
                    assert torch.isnan(got[nan]).all() and torch.equal(got[~nan], clean[~nan]), (which, part, t)


def test_queries_that_are_not_finite():
    for news in (1, 3, 40):
        cache, table, q = setup([90, 0], [news, 1], 4, 2, 128, 16, seed=5)
        args = (dev(starts([news, 1])), dev([90, 0]), dev(table), news)
        clean = binding.kv_attention_u4(q, cache, *args)
        q[news - 1, 1, 7], q[0, 3, 0], q[news, 2, 2] = float("inf"), float("nan"), float("nan")
        got = binding.kv_attention_u4(q, cache, *args)
        bad = torch.zeros(news + 1, 4, dtype=torch.bool, device="cuda")
        bad[news - 1, 1] = bad[0, 3] = True
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad]) and (got[news] == 0).all()


def test_tokens_of_one_value_and_of_zeros():
    """Scale 0 for keys, for values and for both: such tokens count with their offset."""
    cache, table, q = setup([70, 40], [1, 20], 4, 2, 128, 16, seed=9)
    for i in (2, 3):
        cache[i][:, :, 0::3, 0] = 0
        cache[i][:, :, 1::5] = 0
    for news in ([1, 20], [20, 1]):
        got = binding.kv_attention_u4(q, cache, dev(starts(news)), dev([70, 40]), dev(table), 20)
        ref, tol = reference(q, cache, table, [70, 40], news, 0, 128 ** -0.5)
        assert ((got.double() - ref).abs() <= tol).all()


def test_output_pitch_and_stream():
    cache, table, q = setup([90, 33], [2, 1], 8, 2, 128, 16)
    stream = torch.cuda.Stream()
    big = torch.full((3, 8 * 128 + 64), 7.0, device="cuda", dtype=torch.float16)
    out = big[:, :1024].view(3, 8, 128)
    cu, lens, tb = dev([0, 2, 3]), dev([90, 33]), dev(table)
    torch.cuda.synchronize()
    binding.kv_attention_u4(q, cache, cu, lens, tb, 2, out=out, stream=stream)
    stream.synchronize()
    ref, tol = reference(q, cache, table, [90, 33], [2, 1], 0, 128 ** -0.5)
    assert ((out.double() - ref).abs() <= tol).all() and (big[:, 1024:] == 7.0).all()


@pytest.mark.parametrize("news", [1, 40])
def test_captured_into_a_graph(news):
    cache, table, q = setup([9000], [news], 8, 2, 128, 16)
    cu, lens, tb = dev([0, news]), dev([9000]), dev(table)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        binding.kv_attention_u4(q, cache, cu, lens, tb, news, out=out)      # scratch exists before the capture
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.kv_attention_u4(q, cache, cu, lens, tb, news, out=out)
    want = out.clone()
    for L in (5000, 60, 9000):          # lengths are read when the graph runs
        lens.fill_(L)
        graph.replay()
        torch.cuda.synchronize()
        ref, tol = reference(q, cache, table, [L], [news], 0, 128 ** -0.5)
        assert ((out.double() - ref).abs() <= tol).all()
    assert torch.equal(out, want)


@pytest.mark.parametrize("news", [1, 40])
def test_bad_indices_are_reported_and_not_followed(news):
    cache, table, q = setup([64], [news], 4, 1, 64, 16)
    pages = cache[0].shape[0]
    for bad in (pages, -1, 2 ** 31 - 1):
        t = dev(table)
        t[0, 2] = bad
        binding.kv_attention_u4(q, cache, dev([0, news]), dev([64]), t, news)
        assert binding.gemm_last_device_status() == 6
    for cu, L, bound in (([0, news], -5, news), ([0, news], 10 ** 9, news), ([1, 0], 64, news), ([0, news + 1], 64, news + 1)):
        t = dev(np.where(table < 0, 0, table))
        binding.kv_attention_u4(q, cache, dev(cu), dev([L]), t, bound)
        assert binding.gemm_last_device_status() == 6


def test_rows_behind_the_last_sequence_stay():
    for news in ([1, 1], [30, 2]):
        cache, table, q = setup([90, 33], [40, 0], 8, 2, 64, 16)
        out = torch.full_like(q, 7.0)
        binding.kv_attention_u4(q, cache, dev(starts(news)), dev([90, 33]), dev(table), max(news), out=out)
        assert (out[sum(news):] == 7).all() and not (out[:sum(news)] == 7).all(-1).any()


def test_write_then_attend():
    """Cache written token by token, then read by the attention: the chain a decoder runs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    heads, dim, page, n = 2, 128, 16, 50
    table, pages = make_table([n], page)
    cache = binding.kv_cache_u4(pages, heads, page, dim)
    qkv = torch.randn(n, 8 + 2 * heads, dim, generator=g, device="cuda").half()
    tb = dev(table)
    outs = []
    for lo, hi in [(0, 20), (20, 21), (21, 22), (22, 40), (40, 50)]:
        rows, cu = qkv[lo:hi], dev([0, hi - lo])
        binding.kv_append_u4(cache, rows[:, 8:8 + heads], rows[:, 8 + heads:], cu, dev([lo]), tb, hi - lo)
        out = binding.kv_attention_u4(rows[:, :8], cache, cu, dev([hi]), tb, hi - lo)
        ref, tol = reference(rows[:, :8], cache, table, [hi], [hi - lo], 0, dim ** -0.5)
        assert ((out.double() - ref).abs() <= tol).all()
        outs.append(out)
    # and against attention over the unquantised keys and values: a value is off by up to a thirtieth of its row's range, 0.1 of
    # a normal value's size in the mean of squares (range 5.2 / 15 / sqrt(12)), keys and values each
    k, v = qkv[:, 8:8 + heads].double(), qkv[:, 8 + heads:].double()
    sc = torch.einsum("nhgd,thd->nhgt", qkv[:, :8].double().view(n, heads, -1, dim), k) * dim ** -0.5
    sc = sc.masked_fill(torch.triu(torch.ones(n, n, device="cuda", dtype=torch.bool), 1)[:, None, None], -math.inf)
    full = torch.einsum("nhgt,thd->nhgd", sc.softmax(3), v).reshape(n, 8, dim)
    assert (torch.cat(outs).double() - full).norm() / full.norm() < 0.25


def test_refusals():
    cache, table, q = setup([20], [1], 4, 2, 64, 16)
    cu, lens, tb = dev([0, 1]), dev([20]), dev(table)
    for bad in (q.float(), q[..., :32], q[0]):
        with pytest.raises((TypeError, ValueError)):
            binding.kv_attention_u4(bad, cache, cu, lens, tb, 1)
    for kw in (dict(window=-1), dict(softmax_scale=-1.0)):
        with pytest.raises(binding.GemmError):
            binding.kv_attention_u4(q, cache, cu, lens, tb, 1, **kw)
    with pytest.raises(binding.GemmError):
        binding.kv_attention_u4(q[:, :3].contiguous(), cache, cu, lens, tb, 1)
    with pytest.raises((TypeError, ValueError)):
        binding.kv_attention_u4(q, binding.kv_cache_s8(4, 2, 16, 64), cu, lens, tb, 1)
