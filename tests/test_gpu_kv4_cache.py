"""The 4-bit key/value cache: writing and reading back against the definition.

Its arithmetic is FP32 with IEEE operations, so what is read back is compared for equality with the same
operations in numpy, and with the 64-bit inputs: within half a step, and what the scale's rounding to
binary16 (2^-11 of it, fifteen times) and the result's (2^-11) leave."""
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


def held(x):
    """Rows of binary16 as the cache gives them back, with scale and offset."""
    f = np.float32
    bad = ~np.isfinite(x).all(-1, keepdims=True)    # such a row is NaN as a whole
    x = np.where(bad, f(0), x.astype(f))
    low, high = x.min(-1), x.max(-1)
    step = ((high - low) / f(15)).astype(np.float16)
    step = np.where(low + f(15) * step.astype(f) >= f(65520), np.nextafter(step, np.float16(0)), step)
    s = step.astype(f)
    inv = np.where(s > 0, f(1) / np.where(s > 0, s, f(1)), f(0)).astype(f)
    code = np.minimum(np.rint((x - low[..., None]) * inv[..., None]), 15)
    return np.where(bad, np.float16(np.nan), (low[..., None] + code * s[..., None]).astype(np.float16)), step, low


@pytest.mark.parametrize("page,heads,dim", [(16, 1, 64), (16, 8, 128), (32, 3, 256), (64, 8, 128), (128, 2, 64), (128, 5, 256)])
def test_append_and_read(page, heads, dim):
    """Prompts of several lengths, zero among them, then token after token: values at every size."""
    g = np.random.default_rng(3)
    final = [70, 0, 133, 20, 259]
    table, pages = make_table(final, page)
    cache, tb = binding.kv_cache_u4(pages, heads, page, dim), dev(table)
    done, kept = [0] * 5, [[] for _ in range(5)]
    for new in ([30, 0, 1, 20, 200], [1, 0, 100, 0, 1], [39, 0, 32, 0, 58]):
        cu = starts(new)
        rows = (g.standard_normal((cu[-1], 3 * heads, dim)) * np.exp(3 * g.standard_normal((cu[-1], 3 * heads, 1)))).astype(np.float16)
        x = torch.from_numpy(rows).cuda()
        binding.kv_append_u4(cache, x[:, :heads], x[:, heads:2 * heads], dev(cu), dev(done), tb, max(new))
        for b in range(5):
            kept[b].append(rows[cu[b]:cu[b + 1], :2 * heads])
        done = [a + n for a, n in zip(done, new)]
    want = [np.concatenate(v) for v in kept]
    for first, count in (([0] * 5, final), ([69, 0, 16, 0, 100], [1, 0, 100, 20, 159])):
        k, v = binding.kv_read_u4(cache, dev(starts(count)), dev(first), tb, max(count), tokens=sum(count))
        rows = np.concatenate([w[f:f + n] for w, f, n in zip(want, first, count)])
        for got, x in ((k, rows[:, :heads]), (v, rows[:, heads:])):
            back, step, _ = held(x)
            assert np.array_equal(got.cpu().numpy(), back, equal_nan=True)
            fine = np.isfinite(x).all(-1)
            assert fine.mean() > 0.5 and np.isfinite(back[fine]).all()
            s, x64, back = step.astype(np.float64)[fine][..., None], x[fine].astype(np.float64), back[fine]
            assert (np.abs(back.astype(np.float64) - x64) <= s * (0.5 + 15 * 2.0 ** -11) + 2.0 ** -11 * np.abs(x64) + 15 * 2.0 ** -25 + 2.0 ** -25).all()


def test_rows_at_their_edges():
    """Rows of one value, zeros, the largest and the smallest binary16, and rows with what is not finite."""
    heads, dim, page = 2, 64, 16
    g = np.random.default_rng(4)
    x = g.standard_normal((12, heads, dim)).astype(np.float16)
    x[0] = 0
    x[1] = 3.25
    x[2] = -0.0
    x[3, :, 0::2], x[3, :, 1::2] = 65504, -65504
    x[4] = (g.integers(0, 5, (heads, dim)) * 2.0 ** -24).astype(np.float16)
    x[5, :, 7] = 60000
    x[6, 0, 5], x[7, 1, 9], x[8, 0, 63] = np.nan, np.inf, -np.inf
    table, pages = make_table([12], page)
    cache, tb, t = binding.kv_cache_u4(pages, heads, page, dim), dev(table), torch.from_numpy(x).cuda()
    binding.kv_append_u4(cache, t, t, dev([0, 12]), dev([0]), tb, 12)
    got = binding.kv_read_u4(cache, dev([0, 12]), dev([0]), tb, 12, tokens=12)[1].cpu().numpy()
    bad = np.zeros((12, heads), dtype=bool)
    bad[6, 0] = bad[7, 1] = bad[8, 0] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    assert np.array_equal(got[~bad], held(x)[0][~bad])


def test_tokens_do_not_depend_on_the_call():
    heads, dim, page, n = 3, 128, 32, 90
    x = torch.randn(n, 2, heads, dim, device="cuda").half()
    table, pages = make_table([n], page)
    tb = dev(table)
    whole, parts = binding.kv_cache_u4(pages, heads, page, dim), binding.kv_cache_u4(pages, heads, page, dim)
    binding.kv_append_u4(whole, x[:, 0], x[:, 1], dev([0, n]), dev([0]), tb, n)
    for lo, hi in ((0, 33), (33, 34), (34, 64), (64, 90)):
        binding.kv_append_u4(parts, x[lo:hi, 0], x[lo:hi, 1], dev([0, hi - lo]), dev([lo]), tb, hi - lo)
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    # and pages that nobody asked for are as they were
    other = [p for p in range(pages) if p not in table[0]]
    assert all((t[other] == 0).all() for t in whole)


def test_bad_counts_and_pages_are_reported_and_not_followed():
    heads, dim, page = 2, 64, 16
    table, pages = make_table([40], page)
    x = torch.randn(40, heads, dim, device="cuda").half()
    cache = binding.kv_cache_u4(pages, heads, page, dim)
    before = [t.clone() for t in cache]
    for bad in (pages, -1, 2 ** 31 - 1):
        t = dev(table)
        t[0, :] = bad
        binding.kv_append_u4(cache, x, x, dev([0, 40]), dev([0]), t, 40)
        assert binding.gemm_last_device_status() == 6
        binding.kv_read_u4(cache, dev([0, 40]), dev([0]), t, 40, tokens=40)
        assert binding.gemm_last_device_status() == 6
    ok = dev(np.where(table < 0, 0, table))
    for cu, past, most in (([0, 41], 0, 64), ([0, 4], -3, 4), ([0, 4], 10 ** 9, 4), ([4, 0], 0, 4), ([-8, 2], 0, 16)):
        binding.kv_append_u4(cache, x[:0 + 2], x[:2], dev(cu), dev([past]), ok, most)
        assert binding.gemm_last_device_status() == 6, (cu, past)
    for a, b in zip(cache[:2], before[:2]):     # what was written are the two rows that exist, at most
        assert (a != b).any(-1).sum() <= 2 * heads


def test_captured_into_a_graph():
    heads, dim, page = 2, 128, 16
    table, pages = make_table([64], page)
    cache, tb, past = binding.kv_cache_u4(pages, heads, page, dim), dev(table), dev([5])
    x = torch.randn(1, heads, dim, device="cuda").half()
    cu, out = dev([0, 1]), tuple(torch.empty(1, heads, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.kv_append_u4(cache, x, x, cu, past, tb, 1)
            binding.kv_read_u4(cache, cu, past, tb, 1, out=out)
    for at in (5, 6, 63):
        past.fill_(at)
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = held(x.cpu().numpy())[0]
        assert np.array_equal(out[0].cpu().numpy(), want) and np.array_equal(out[1].cpu().numpy(), want)


def test_refusals():
    cache = binding.kv_cache_u4(4, 2, 16, 64)
    x = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    cu, past, table = dev([0, 4]), dev([0]), dev([[0, 1]])
    for c in (binding.kv_cache_s8(4, 2, 16, 64), cache[:3], (cache[0], cache[1], cache[2][:, :, :, :1].contiguous(), cache[3]),
              (cache[0], cache[1][:2], cache[2], cache[3]), (cache[0], cache[1], cache[2].float(), cache[3].float())):
        with pytest.raises((TypeError, ValueError)):
            binding.kv_append_u4(c, x, x, cu, past, table, 4)
    with pytest.raises(ValueError):
        binding.kv_append_u4(cache, x[:, :1], x[:, :1], cu, past, table, 4)
    with pytest.raises(binding.GemmError):
        binding.kv_append_u4(binding.kv_cache_u4(4, 2, 24, 64), x, x, cu, past, table, 4)
