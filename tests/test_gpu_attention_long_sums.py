"""Attention of long rows on the tensor cores: what an accumulator cuts off must not add up over the tokens.

An instruction of 16 tokens cuts off up to two units of 2^-24 of what the accumulator holds, towards zero. Sums go on from almost nothing
every 16384 tokens, so that a result shrinks by up to 16384 / 16 * 2 * 2^-24 = 1.22e-4 (4-bit values in two tiles: the second one's products are small,
and cut off as much of the accumulator again, 2.44e-4). The other roundings have no sign: 3e-4 a value, 2e-6 over the 2e4 values and more that are compared,
so that 1e-5 is allowed for them. Single values are held against 64 bits with the attention tests' bound and these 1.22e-4 or 2.44e-4
in place of what it allows a token."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv4_attention import values
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def compare(got, q, k, v, pos, window, scale, top, cut, q_bits=0.0):
    """Rows q [n, g, dim] at positions pos over tokens of 64-bit k, v; top: the most a value of a token could be, or |v|."""
    num = den = 0.0
    for lo in range(0, len(pos), 64):
        x, p = q[lo:lo + 64].double(), pos[lo:lo + 64]
        sc = torch.einsum("ngd,td->ngt", x, k) * scale
        mag = (torch.einsum("ngd,td->ngt", x.abs(), k.abs()) * scale).amax(2, keepdim=True)
        tok = torch.arange(k.shape[0], device="cuda")[None]
        hidden = tok > p[:, None]
        if window:
            hidden = hidden | (tok <= p[:, None] - window)
        w = torch.softmax(sc.masked_fill(hidden[:, None], -math.inf), dim=2)
        ref, mass = torch.einsum("ngt,td->ngd", w, v), torch.einsum("ngt,td->ngd", w, top)
        n = hidden.logical_not().sum(1).max().item()
        # weights to binary16, scores in FP32 twice, FP32 sums; the rest as above
        tol = (2.0 ** -11 + 2 * 2.0 ** -20 * mag + 4e-6 + cut) * mass + 2.0 ** -11 * ref.abs() + 2.0 ** -25 + n * 2.0 ** -32 * top.max()
        err = got[lo:lo + 64].double() - ref
        assert (err.abs() <= tol).all(), "worst %.3g x bound" % (err.abs() / tol).max().item()
        num, den = num + (err * ref).sum().item(), den + (ref * ref).sum().item()
    return num / den


def prompt(lens, q_heads, kv_heads, dim, mean=0.0, rise=0.0, window=0, causal=True, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q, k, v = (torch.randn(sum(lens), h, dim, generator=g, device="cuda").half() for h in (q_heads, kv_heads, kv_heads))
    v += mean
    if rise:          # scores grow along the sequence: sums put by are scaled down later
        at = torch.cat([torch.linspace(0, rise, n, device="cuda") for n in lens])
        q[..., 0] = dim ** 0.5
        k[..., 0] = at[:, None].half()
    args = (q, k, v, dev(starts(lens)), max(lens))
    got = binding.attention_fp16(*args, window=window, causal=causal)
    assert torch.equal(got, binding.attention_fp16(*args, window=window, causal=causal))
    shrink, at, group = [], 0, q_heads // kv_heads
    for n in lens:
        rows = torch.unique(torch.cat([torch.arange(max(0, n - 150), n), torch.randint(0, n, (100,))])).cuda()
        for h in (0, kv_heads - 1):
            mine = slice(h * group, h * group + group)
            kk, vv = k[at:at + n, h].double(), v[at:at + n, h].double()
            shrink.append(compare(got[at + rows][:, mine], q[at + rows][:, mine], kk, vv, rows if causal else torch.full_like(rows, n - 1), window,
                                  dim ** -0.5, vv.abs(), 1.22e-4))
        at += n
    return shrink


def chunk(length, new, kv_heads, group, dim, mean=0.0, rise=0.0, window=0, page=64):
    g = torch.Generator(device="cuda")
    g.manual_seed(length + dim)
    pages = -(-length // page)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    cache = list(binding.kv_cache_u4(pages, kv_heads, page, dim))
    for i in range(2):
        cache[i].random_(0, 256, generator=g)
        step = 0.1 + 0.1 * torch.rand(pages, kv_heads, page, generator=g, device="cuda")
        if rise and i == 0:
            step[table[0].long()] *= torch.linspace(0.1, rise, pages, device="cuda")[:, None, None]
        cache[2 + i] = torch.stack((step, -7.5 * step + (mean if i else 0.0)), dim=3).half()
    q = torch.randn(new, kv_heads * group, dim, generator=g, device="cuda").half()
    args = (q, tuple(cache), dev([0, new]), dev([length]), table, new)
    got = binding.kv_attention_u4(*args, window=window)
    assert torch.equal(got, binding.kv_attention_u4(*args, window=window))
    shrink, slots = [], table[0].long()
    pos = length - new + torch.arange(new, device="cuda")
    for h in (0, kv_heads - 1):
        (kk, _), (vv, top) = ([x.reshape(-1, dim)[:length] for x in values(cache[i][slots, h], cache[2 + i][slots, h])] for i in range(2))
        mine = slice(h * group, h * group + group)
        shrink.append(compare(got[:, mine], q[:, mine], kk, vv, pos, window, dim ** -0.5, top, 2.44e-4))
    return shrink


@pytest.mark.parametrize("mean", [0.0, 0.3, 3.0])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_no_shrinking(mean, dim):
    for s in prompt([131072], 2, 2, dim, mean=mean):
        assert abs(s) <= 1.22e-4 + 1e-5
    for s in chunk(200000, 300, 24, 1, dim, mean=mean):
        assert abs(s) <= 2.44e-4 + 1e-5


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts(dim):
    """Lengths around a sum's end, several row tiles of all lengths per CTA, scores that rise by many powers of two, windows."""
    prompt([16385, 16384, 50], 2, 2, dim)
    prompt([32768, 32833, 300], 4, 1, dim, rise=40.0, seed=1)
    prompt([49000], 3, 1, dim, rise=4.0, window=33000, seed=2)
    prompt([36000, 17000], 2, 1, dim, causal=False, mean=1.0, seed=3)
    prompt([16500], 100, 2, dim, rise=300.0, seed=4)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("length,new,kv_heads,window", [(16384, 300, 80, 0), (16385, 260, 80, 0), (33000, 300, 80, 0), (70000, 300, 32, 0),
                                                        (300000, 40, 4, 0), (150000, 300, 20, 0), (70000, 300, 80, 40000)])
def test_chunks(length, new, kv_heads, window, dim):
    """The same over 4-bit tokens, also where they are divided over CTAs."""
    chunk(length, new, kv_heads, 1 if kv_heads == 80 else 4, dim, rise=3.0, window=window)


def test_values_at_the_end_of_the_range():
    """Sums put by stay in binary16 where results do; infinities and NaN pass."""
    n = 20000
    q, k = (torch.randn(n, 1, 64, device="cuda").half() for _ in range(2))
    v = torch.full((n, 1, 64), 65504.0, device="cuda", dtype=torch.float16)
    v[:, 0, 1] = 2.0 ** -24
    v[:, 0, 2] *= -1
    got = binding.attention_fp16(q, k, v, dev([0, n]), n)
    assert (got[..., 0] >= 65440).all() and torch.isfinite(got).all() and torch.equal(got[..., 2], -got[..., 0])
    assert (got[..., 1] == 2.0 ** -24).all()
    k.zero_()      # all weights alike: an infinity keeps its own
    v[100, 0, 3], v[300, 0, 4] = float("inf"), float("nan")
    v[17000, 0, 5] = float("-inf")
    got = binding.attention_fp16(q, k, v, dev([0, n]), n)
    assert (got[100:, 0, 3] == float("inf")).all() and torch.isfinite(got[:100, 0, 3]).all()
    assert torch.isnan(got[300:, 0, 4]).all() and (got[17000:, 0, 5] == float("-inf")).all() and torch.isfinite(got[:17000, 0, 5]).all()


def test_rows_behind_the_last_sequence_stay():
    n = 17000
    q, k, v = (torch.randn(n + 100, h, 128, device="cuda").half() for h in (6, 2, 2))
    out = torch.full((n + 100, 6, 128), 7.0, device="cuda", dtype=torch.float16)
    binding.attention_fp16(q, k, v, dev([0, n]), n, out=out)
    assert (out[n:] == 7).all()


def test_two_streams_and_graphs():
    """Sums are put by in a call's own results: calls side by side do not meet, and a capture needs no call before it."""
    n = 20000
    sets = [[torch.randn(n, h, 64, device="cuda").half() for h in (2, 1, 1)] for _ in range(2)]
    cu = dev([0, n])
    want = [binding.attention_fp16(*s, cu, n) for s in sets]
    outs, graphs, streams = [torch.empty_like(w) for w in want], [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, out, stream in zip(sets, outs, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            binding.attention_fp16(*s, cu, n, out=out)
        graphs.append(graph)
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
