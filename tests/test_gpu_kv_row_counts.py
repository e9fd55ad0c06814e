"""Row counts on the device that go beyond the packed arrays: what lies behind the rows a call was given is
neither read nor written, and the status word says so.

Every array here is the front of a larger one, so that a kernel that followed the counts would still stay inside
its allocation: the rows behind are guards."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference, setup
from test_gpu_kv_cache import dev, make_table

pytestmark = pytest.mark.gpu
GUARD = 64


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("cu", [[0, 20, 45], [0, 20, 60], [0, 45, 50], [0, 41, 41], [44, 50, 60]])
def test_append_reads_no_row_behind_the_last(cu):
    """Rows behind the last are NaN: had one been read, its page's scale would be NaN."""
    heads, dim, page, rows = 2, 64, 16, 40
    table, pages = make_table([64, 64], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    big = torch.full((rows + GUARD, heads, dim), float("nan"), device="cuda", dtype=torch.float16)
    big[:rows] = 1.0
    binding.kv_append_s8(cache, big[:rows], big[:rows], dev(cu), dev([0, 0]), dev(table), 64)
    assert binding.gemm_last_device_status() == 6
    for scale in cache[2:]:
        assert torch.isfinite(scale).all()
    seen = sum(max(0, min(b, rows) - a) for a, b in zip(cu, cu[1:]))
    for codes in cache[:2]:
        assert int((codes != 0).sum()) == seen * heads * dim      # every row there is, and none else


@pytest.mark.parametrize("cu", [[0, 20, 45], [0, 20, 60], [0, 45, 50], [0, 41, 41], [44, 50, 60]])
def test_read_writes_no_row_behind_the_last(cu):
    heads, dim, page, rows = 2, 64, 16, 40
    table, pages = make_table([64, 64], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    x = torch.randn(128, heads, dim, device="cuda").half()
    binding.kv_append_s8(cache, x, x, dev([0, 64, 128]), dev([0, 0]), dev(table), 64)
    whole = binding.kv_read_s8(cache, dev([0, 64, 128]), dev([0, 0]), dev(table), 64, tokens=128)
    big = [torch.full((rows + GUARD, heads, dim), 7.0, device="cuda", dtype=torch.float16) for _ in range(2)]
    binding.kv_read_s8(cache, dev(cu), dev([0, 0]), dev(table), 64, out=(big[0][:rows], big[1][:rows]))
    assert binding.gemm_last_device_status() == 6
    for got, src in zip(big, whole):
        want = torch.full_like(got, 7.0)
        for b in range(2):
            n = max(0, min(cu[b + 1], rows) - cu[b])
            want[cu[b]:cu[b] + n] = src[64 * b:64 * b + n]
        assert torch.equal(got, want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news,cu,rows", [([3, 2], [0, 3, 5], 4), ([3, 2], [0, 3, 5], 3), ([60, 70], [0, 60, 130], 100),
                                          ([60, 3], [0, 60, 63], 61), ([3, 60], [0, 3, 63], 2)])
def test_attention_stays_inside_its_rows(dim, news, cu, rows):
    lens = [100, 130]
    cache, table, q = setup(lens, news, 4, 1, dim, 16)
    full = torch.full((cu[-1] + GUARD, 4, dim), 7.0, device="cuda", dtype=torch.float16)
    binding.kv_attention_s8(q[:rows], cache, dev(cu), dev(lens), dev(table), max(news), out=full[:rows])
    assert binding.gemm_last_device_status() == 6
    assert (full[rows:] == 7.0).all()
    if rows >= cu[1]:                  # the first sequence is all there: its result stands
        ref, tol = reference(q, cache, table, lens, news, 0, dim ** -0.5)
        assert ((full[:cu[1]].double() - ref[:cu[1]]).abs() <= tol[:cu[1]]).all()


def test_counts_that_fit_report_nothing():
    cache, table, q = setup([100, 130], [3, 60], 4, 1, 64, 16)
    binding.kv_attention_s8(q, cache, dev([0, 3, 63]), dev([100, 130]), dev(table), 60)
    k, v = binding.kv_read_s8(cache, dev([0, 3, 63]), dev([1, 60]), dev(table), 60, tokens=63)
    binding.kv_append_s8(cache, k, v, dev([0, 3, 63]), dev([1, 60]), dev(table), 60)
    assert binding.gemm_last_device_status() == 0
