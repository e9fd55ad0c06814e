"""kv_read_s8 without a token count, on a stream of its own: cu is read in that stream's order."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_cache import dev, make_table

pytestmark = pytest.mark.gpu


def test_count_comes_from_the_stream():
    heads, dim, page, n = 2, 64, 16, 40
    table, pages = make_table([n], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    x = torch.randn(n, heads, dim, device="cuda").half()
    cu, tb, zero, real = dev([0, 0]), dev(table), dev([0]), dev([0, n])
    binding.kv_append_s8(cache, x, x, real, zero, tb, n)
    want = binding.kv_read_s8(cache, real, zero, tb, n, tokens=n)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)          # some 25 ms
        cu.copy_(real)
    got = binding.kv_read_s8(cache, cu, zero, tb, n, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
