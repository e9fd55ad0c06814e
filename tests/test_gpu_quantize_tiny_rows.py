"""FP32 rows whose largest value is so small that T / amax leaves the type: codes and scales by the definition.

The codes against x * (T / amax) in 64 bits: three FP32 roundings of a value of at most T, and half a step; the scale
is the FP32 quotient (below the normal range a multiple of 2^-149)."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_linear import rng, unpack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,top", [("s8", 127.0), ("s4", 7.0)])
@pytest.mark.parametrize("K", [64, 1024, 40000])
@pytest.mark.parametrize("size", [1e-18, 5e-20, 1e-30, 3.8e-37, 3.6e-37, 1.3e-38, 1e-38, 1e-41, 1e-44])
def test_tiny_rows(prec, top, K, size):
    # (made on the host in 64 bits: values below the normal range come out rounded once)
    x = torch.randn(5, K, generator=torch.Generator().manual_seed(K), dtype=torch.float64)
    x = (x / x.abs().amax(1, keepdim=True) * size).float()
    x[3] = 1.0 / 3                               # an ordinary row among them
    q, s = binding.gemm_quantize_rows(x.cuda(), prec)
    codes = (q.to(torch.int32) if prec == "s8" else unpack(q).to(torch.int32)).cpu().double()
    amax = x.double().abs().amax(1)
    assert torch.equal(s.cpu(), (amax / top).float())      # (one rounding of an exact quotient, or its double rounding: equal here)
    want = x.double() * (top / amax)[:, None]
    assert ((codes - want).abs() <= 0.5 + 3 * top * 2.0 ** -24).all()
    assert (codes.abs().amax(1) == top).all()


def test_rows_that_are_not_a_number_have_no_codes():
    x = torch.randn(4, 512, generator=rng(2), device="cuda")
    x[1, 3], x[2, 5] = float("nan"), float("inf")
    for dtype in (torch.float16, torch.float32):
        q, s = binding.gemm_quantize_rows(x.to(dtype), "s8")
        assert (q[1:3] == 0).all() and torch.isnan(s[1]) and torch.isinf(s[2]) and (q[[0, 3]] != 0).any()
