"""Infinite sums through every activation: what the formula gives in 64 bits, in kind and sign."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_linear import activate, operands

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    binding.gemm_set_kernel_family(0)
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("act", list(binding.ACTIVATIONS))
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("M,N", [(1, 600), (40, 1200), (300, 520), (1100, 1208)])
def test_infinite_sums(act, dtype, M, N):
    if M == 1100:
        binding.gemm_set_kernel_family(2)
    for prec in ("fp16", "s8", "s4"):
        A, B, rs, cs = operands(prec, M, N, 512, 1)
        bias = torch.zeros(N, device="cuda")
        bias[::3], bias[1::3], bias[2::3] = math.inf, -math.inf, 1.0
        call = {"fp16": binding.gemm_fp16_linear, "s8": binding.gemm_s8_linear, "s4": binding.gemm_s4_linear}[prec]
        got = call(A, B, *(() if rs is None else (rs, cs)), bias=bias, activation=act, out_dtype=dtype)
        want = activate(bias.double(), act)
        for j in range(2):
            w, x = want[j], got[:, j::3]
            assert torch.isnan(x).all() if math.isnan(w) else (x == w.item()).all()
        assert torch.isfinite(got[:, 2::3]).all()


@pytest.mark.parametrize("act", list(binding.ACTIVATIONS))
def test_large_finite_sums(act):
    """Where squares and exponentials overflow the result still is x, or zero."""
    A, B, _, _ = operands("fp16", 9, 600, 64, 1)
    big = torch.tensor([50.0, 90.0, 1e4, 1e10, 1e20, 3e38], device="cuda").repeat(100)
    for sign in (1.0, -1.0):
        got = binding.gemm_fp16_linear(A * 0, B, bias=sign * big, activation=act, out_dtype=torch.float32)
        want = sign * big.double() if sign > 0 or act == "none" else torch.zeros_like(big).double()
        assert ((got.double() - want).abs() <= 1e-6 * want.abs() + 1e-15).all()
