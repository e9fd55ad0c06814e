"""Matrices whose rows are one row broadcast, or overlap otherwise, are refused before anything is launched: their
pitch of 0 would be taken for the dense one and the rows read (or written) behind the single row there is."""
import pytest
import torch

from paper_2608_10103_b200 import binding

pytestmark = pytest.mark.gpu
M, N, K = 8, 64, 32


def overlapping(cols, dtype):
    one = torch.ones(1, cols, device="cuda", dtype=dtype)
    yield one.expand(M, cols)
    yield torch.ones(M * cols, device="cuda", dtype=dtype).as_strided((M, cols), (cols // 2, 1))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_refused(dtype):
    A = torch.ones(M, K, device="cuda", dtype=torch.float16)
    B = torch.ones(N, K, device="cuda", dtype=torch.float16)
    for x in overlapping(K, dtype):
        for prec in ("s8", "s4"):
            with pytest.raises(ValueError, match="overlap"):
                binding.gemm_quantize_rows(x, prec)
    for r in overlapping(N, dtype):
        with pytest.raises(ValueError, match="overlap"):
            binding.gemm_fp16_linear(A, B, residual=r, out_dtype=dtype)
        with pytest.raises(ValueError, match="overlap"):
            binding.gemm_fp16_linear(A, B, C=r)
    q = torch.ones(M, K, device="cuda", dtype=torch.int8)
    w = torch.ones(N, K, device="cuda", dtype=torch.int8)
    one = torch.ones(N, device="cuda")
    for r in overlapping(N, dtype):
        with pytest.raises(ValueError, match="overlap"):
            binding.gemm_s8_linear(q, w, one[:M], one, residual=r, out_dtype=dtype)


def test_one_row_may_have_any_pitch():
    x = torch.randn(1, K, device="cuda").half()
    q, s = binding.gemm_quantize_rows(x.as_strided((1, K), (0, 1)), "s8")
    q2, s2 = binding.gemm_quantize_rows(x, "s8")
    assert torch.equal(q, q2) and torch.equal(s, s2)
