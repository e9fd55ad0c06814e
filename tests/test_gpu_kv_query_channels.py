"""Queries with one channel far above the others, which the two attention kernels hold differently; bound as for small
weights, with the term for a row of q of one scale where the few-rows kernel runs."""
import pytest

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import setup
from test_gpu_kv_cache import dev
from test_gpu_kv_small_weights import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 2, 40])
def test_one_channel_far_above_the_others(new, dim):
    """The few-rows kernel holds a row of q with one scale, the tile kernel as it is: both against the definition."""
    cache, table, q = setup([700], [new], 8, 2, dim, 32, spread=0.3, seed=8)
    q[..., 11] *= 64
    cache[0][..., 11] = cache[0][..., 11] // 16        # (the keys' channel is small, as norms leave it)
    got = binding.kv_attention_s8(q, cache, dev([0, new]), dev([700]), dev(table), new)
    ref, tol, _ = reference(q, cache, table, [700], [new], dim ** -0.5, new * 4 <= (16 if dim == 256 else 32))
    assert (ref.abs() > tol).any()                     # (the bound is wide here: zeros must not pass)
    assert ((got.double() - ref).abs() <= tol).all()
    assert binding.gemm_last_device_status() == 0
