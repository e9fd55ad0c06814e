"""Batches whose tables could name very long sequences are served, not refused."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,group", [(1, 4), (3, 4), (8, 4), (20, 4)])
def test_many_sequences_with_wide_tables(new, group):
    """512 sequences, 8 KV heads, tables of a million tokens."""
    batch, heads, dim, page, width = 512, 8, 64, 128, 8192
    g = torch.Generator(device="cuda")
    g.manual_seed(new)
    cache = list(binding.kv_cache_s8(64, heads, page, dim))
    for i in range(2):
        cache[i] = torch.randint(-127, 128, cache[i].shape, generator=g, device="cuda").to(torch.int8)
        cache[2 + i].fill_(0.01)
    table = torch.randint(0, 64, (batch, width), generator=g, device="cuda").to(torch.int32)
    lens = [20 + (7 * b) % 300 for b in range(batch)]
    q = torch.randn(batch * new, heads * group, dim, generator=g, device="cuda").half()
    got = binding.kv_attention_s8(q, tuple(cache), dev([new * b for b in range(batch + 1)]), dev(lens), table, new)
    assert binding.gemm_last_device_status() == 0
    pick = [0, 3, 255, 511]
    ref, tol = reference(torch.cat([q[new * b:new * b + new] for b in pick]), cache, table.cpu().numpy()[pick],
                         [lens[b] for b in pick], [new] * 4, 0, dim ** -0.5)
    got = torch.cat([got[new * b:new * b + new] for b in pick])
    assert ((got.double() - ref).abs() <= tol).all()
