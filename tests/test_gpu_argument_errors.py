"""Numbers that are no integers, or that 32 bits do not hold, are refused with the error Python has for that."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import setup
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.fixture
def calls():
    cache, table, q = setup([20], [2], 4, 2, 64, 16)
    cu, lens, tb, kv = dev([0, 2]), dev([20]), dev(table), q[:, :2].contiguous()
    torch.cuda.synchronize()
    yield {
        "max_new": lambda v: binding.kv_append_s8(cache, kv, kv, cu, dev([18]), tb, v),
        "max_read": lambda v: binding.kv_read_s8(cache, cu, dev([0]), tb, v, tokens=2),
        "tokens": lambda v: binding.kv_read_s8(cache, cu, dev([0]), tb, 2, tokens=v),
        "max_q": lambda v: binding.kv_attention_s8(q, cache, cu, lens, tb, v),
        "window": lambda v: binding.kv_attention_s8(q, cache, cu, lens, tb, 2, window=v),
    }
    binding.gemm_last_device_status()


@pytest.mark.parametrize("name", ["max_new", "max_read", "tokens", "max_q", "window"])
def test_integers(calls, name):
    f = calls[name]
    f(2)
    for wide in (2 ** 32 + 2, 2 ** 31, -2 ** 32 + 2, 2 ** 70, -2 ** 70):
        with pytest.raises(ValueError):
            f(wide)
    for wrong in ("2", 2.0, None if name != "tokens" else [], object()):
        with pytest.raises(TypeError):
            f(wrong)
    f(2)


def test_softmax_scale():
    cache, table, q = setup([20], [2], 4, 2, 64, 16)
    cu, lens, tb = dev([0, 2]), dev([20]), dev(table)
    for wrong in ("0.1", [0.1]):
        with pytest.raises(TypeError):
            binding.kv_attention_s8(q, cache, cu, lens, tb, 2, softmax_scale=wrong)
    for scale in (1e300, -1.0, float("nan")):
        with pytest.raises(binding.GemmError):
            binding.kv_attention_s8(q, cache, cu, lens, tb, 2, softmax_scale=scale)
    binding.kv_attention_s8(q, cache, cu, lens, tb, 2, softmax_scale=1)
