"""Attention over the INT8 cache beside pages whose scale is below 0, which no append leaves: NaN for the queries that see one."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_cache import dev, make_table, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 8, 30, 200])
@pytest.mark.parametrize("which", [2, 3])
def test_negative_scales(dim, rows, which):
    lens, page = [700, 300], 32
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    table, pages = make_table(lens, page)
    cache = binding.kv_cache_s8(pages, 2, page, dim)
    for i in range(2):
        cache[i].copy_(torch.randint(-127, 128, cache[i].shape, generator=g, device="cuda", dtype=torch.int8))
        cache[2 + i].fill_(0.01)
    q = torch.randn(2 * rows, 2, dim, generator=g, device="cuda").half()
    args = (dev(starts([rows, rows])), dev(lens), dev(table), rows)
    for window in (0, 40):
        cache[which].fill_(0.01)
        cache[which][0] = 0.0
        clean = binding.kv_attention_s8(q, cache, *args, window=window)
        at, last = 620, 640       # the page that holds these tokens of the first sequence, of one head
        cache[which][int(table[0, at // page]), 1] = -0.01
        got = binding.kv_attention_s8(q, cache, *args, window=window)
        pos = 700 - rows + torch.arange(rows, device="cuda")
        sees = (pos >= at // page * page) & ((pos - window < last - 1) if window else torch.ones_like(pos, dtype=torch.bool))
        assert torch.isnan(got[:rows, 1][sees]).all()
        got[:rows, 1][sees] = clean[:rows, 1][sees]
        assert torch.equal(got, clean)
        cache[which].fill_(-0.0)  # a zero, whatever its sign
        assert torch.isfinite(binding.kv_attention_s8(q, cache, *args, window=window)).all()
