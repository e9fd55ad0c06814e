"""Pages whose scale is not finite, and queries that are not: what a query does not see leaves its result alone,
whatever is stored there; what it does see makes its result NaN.

The clean results are held against the definition in 64 bits with the bound of the attention tests."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference, setup
from test_gpu_kv_cache import dev, make_table

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def positions(lens, news):
    return torch.cat([torch.arange(L - n, L) for L, n in zip(lens, news)]).cuda()


# (lens, news): within the few-rows kernel (4 heads to a KV head: 32 rows, 16 at 256 d), and row tiles
FEW = [([228], [8]), ([228], [4]), ([130, 228], [1, 2])]
MANY = [([240], [240]), ([900, 300], [60, 100])]


@pytest.mark.parametrize("which,value", [(2, NAN), (2, INF), (3, NAN), (3, INF)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,news", FEW + MANY)
def test_later_pages(lens, news, dim, which, value):
    """The last page of each sequence (and the one that holds its queries' middle)."""
    page = 16
    cache, table, q = setup(lens, news, 4, 1, dim, page)
    ref, tol = reference(q, cache, table, lens, news, 0, dim ** -0.5)
    pos, seq = positions(lens, news), torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(news)).cuda()
    for at in (lambda L, n: (L - 1) // page, lambda L, n: (L - n // 2) // page):
        first = dev([at(L, n) * page for L, n in zip(lens, news)])[seq]
        poisoned = [t.clone() for t in cache]
        for b, (L, n) in enumerate(zip(lens, news)):
            poisoned[which][int(table[b, at(L, n)])] = value
        got = binding.kv_attention_s8(q, poisoned, dev([0] + list(torch.tensor(news).cumsum(0))), dev(lens), dev(table), max(news))
        sees = pos >= first
        assert torch.isnan(got[sees]).all()
        assert ((got.double() - ref).abs() <= tol)[~sees].all()


@pytest.mark.parametrize("which,value", [(2, NAN), (2, INF), (3, NAN), (3, INF)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,news,window", [([228], [4], 20), ([500], [300], 50), ([300, 90], [80, 2], 33)])
def test_pages_behind_the_window(lens, news, window, dim, which, value):
    """A page in the middle of the queries: those in front of it and those whose window has left it."""
    page = 16
    cache, table, q = setup(lens, news, 4, 1, dim, page)
    ref, tol = reference(q, cache, table, lens, news, window, dim ** -0.5)
    pos, seq = positions(lens, news), torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(news)).cuda()
    bad = [(L - n // 2 - window // 2) // page for L, n in zip(lens, news)]
    for b in range(len(lens)):
        cache[which][int(table[b, bad[b]])] = value
    got = binding.kv_attention_s8(q, cache, dev([0] + list(torch.tensor(news).cumsum(0))), dev(lens), dev(table), max(news),
                                  window=window)
    first = dev([j * page for j in bad])[seq]
    sees = (pos >= first) & (pos - window + 1 < first + page)
    assert torch.isnan(got[sees]).all() and sees.any()
    assert ((got.double() - ref).abs() <= tol)[~sees].all()


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("into", ["k", "v"])
def test_a_token_that_is_not_finite(into, value):
    """Written by the cache itself: everything in front of its page stays as it was."""
    n, heads, dim, page, token = 300, 2, 128, 16, 220
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    table, pages = make_table([n], page)
    rows = torch.randn(n, 4 * heads + 2 * heads, dim, generator=g, device="cuda").half()
    q, k, v = rows[:, :8], rows[:, 8:10], rows[:, 10:]
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    binding.kv_append_s8(cache, k, v, dev([0, n]), dev([0]), dev(table), n)
    ref, tol = reference(q, cache, table, [n], [n], 0, dim ** -0.5)
    (k if into == "k" else v)[token, 1, 5] = value
    binding.kv_append_s8(cache, k, v, dev([0, n]), dev([0]), dev(table), n)
    got = binding.kv_attention_s8(q, cache, dev([0, n]), dev([n]), dev(table), n)
    first = token // page * page
    ok = (got.double() - ref).abs() <= tol
    assert ok[:first].all() and ok[:, :4].all() and torch.isnan(got[first:, 4:]).all()
    for lo, count in ((first - 5, 5), (first - 3, 6)):      # the same from the few-rows kernel
        cu, lens = dev([0, count]), dev([lo + count])
        few = binding.kv_attention_s8(q[lo:lo + count], cache, cu, lens, dev(table), count)
        ok = (few.double() - ref[lo:lo + count]).abs() <= tol[lo:lo + count]
        assert ok[:first - lo].all() and ok[:, :4].all() and torch.isnan(few[first - lo:, 4:]).all()
