"""FP32 results of FP16 linear layers keep what an FP32 sum keeps, at every length of K.

A chain of L products is L / 16 accumulations, each cutting off 0.72 units of 2^-24 of an accumulator that has on average
2/3 of its final size: 1.8e-9 L of the result's norm.  K is summed in parts of L = 640, of up to 20 sqrt(K) for
results of a million values and more; adding the parts rounds each at most once, 2e-7 for those there are here."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_linear import operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(1, 4096), (16, 2048), (40, 2048), (100, 3000), (300, 1001), (652, 176), (300, 4096), (1000, 4096), (2500, 2500)])
@pytest.mark.parametrize("K", [64, 632, 640, 648, 1096, 1280, 2048, 2056, 4096, 8192, 16384])
def test_sums(M, N, K):
    A, B, _, _ = operands("fp16", M, N, K, K + M)
    A[:, ::max(1, K // 7)] *= 8                # a few channels above the others
    x = A.double() @ B.double().t()
    got = binding.gemm_fp16_linear(A, B, out_dtype=torch.float32)
    part = 640 if min(M, N) <= 128 or M * N < 2 ** 20 else max(640, min(2048, 20 * math.sqrt(K)))
    assert (got.double() - x).norm() <= (1.8e-9 * min(K, part) + 2e-7) * x.norm()
    assert binding.gemm_last_device_status() == 0
