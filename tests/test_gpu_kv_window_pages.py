"""Table entries behind the window: a serving program gives those pages away, so they may name anything."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference, setup
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,news,window", [([1000], [1], 100), ([1000, 333], [2, 1], 17), ([1000], [60], 100),
                                              ([2000, 700], [300, 40], 130), ([1111], [64], 1)])
def test_entries_behind_the_window_are_not_looked_at(lens, news, window, page, dim):
    cache, table, q = setup(lens, news, 4, 1, dim, page)
    cu = dev([0] + list(torch.tensor(news).cumsum(0)))
    want = binding.kv_attention_s8(q, cache, cu, dev(lens), dev(table), max(news), window=window)
    for b, (L, n) in enumerate(zip(lens, news)):
        table[b, :max(0, L - n - window + 1) // page] = -1 if b == 0 else 2 ** 31 - 1
    got = binding.kv_attention_s8(q, cache, cu, dev(lens), dev(table), max(news), window=window)
    assert binding.gemm_last_device_status() == 0
    assert torch.equal(got, want)
    ref, tol = reference(q, cache, table * (table >= 0) * (table < cache[0].shape[0]), lens, news, window, dim ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()
