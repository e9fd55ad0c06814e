"""Prompt attention: a `causal` that has no truth value raises what asking for it raises."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


class Undecided:
    def __bool__(self):
        raise KeyError("undecided")


def test_causal_without_a_truth_value():
    q = torch.randn(8, 2, 64, device="cuda").half()
    with pytest.raises(KeyError):
        binding.attention_fp16(q, q, q, dev([0, 8]), 8, causal=Undecided())
    with pytest.raises(RuntimeError):
        binding.attention_fp16(q, q, q, dev([0, 8]), 8, causal=torch.ones(2))
    a = binding.attention_fp16(q, q, q, dev([0, 8]), 8, causal=torch.ones(1))
    assert torch.equal(a, binding.attention_fp16(q, q, q, dev([0, 8]), 8, causal=True))
    assert binding.gemm_last_device_status() == 0
