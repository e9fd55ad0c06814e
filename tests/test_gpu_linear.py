"""Linear layers (act(A B^T [* scales] + bias) + residual in the GEMM epilogues) and row quantisation
against the definition in 64 bits.

Tolerance.  With x the sum (scaled) before the bias, e = error of x: 1e-4 sum|a b| + 1e-6 for FP16
operands (the library's bound), 4 roundings of an exact sum for the integer kinds.  The activations'
slopes stay below 1.13, their own error below 1e-6 |x|; bias and residual add a rounding each;
a binary16 result one rounding of 2^-11 (2^-25 below its normal range)."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(autouse=True)
def _clean_state():
    binding.gemm_set_config_override(0, 0, 0)
    binding.gemm_set_kernel_family(0)
    yield
    binding.gemm_set_config_override(0, 0, 0)
    binding.gemm_set_kernel_family(0)
    binding.gemm_set_s4_scheme(0)
    binding.gemm_set_swap_ab(0)
    assert binding.gemm_last_device_status() == 0


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def unpack(p):
    p = p.long()
    return torch.stack((((p & 15) ^ 8) - 8, ((p >> 4) ^ 8) - 8), dim=2).flatten(1)


def activate(x, name):
    if name == "relu":
        return x.clamp(min=0)
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if name == "silu":
        return x / (1 + torch.exp(-x))
    return x


def operands(prec, M, N, K, seed):
    g = rng(seed)
    if prec == "fp16":
        A = torch.randn(M, K, generator=g, device="cuda").half()
        B = (torch.randn(N, K, generator=g, device="cuda") / math.sqrt(K)).half()
        return A, B, None, None
    if prec == "s8":
        A = torch.randint(-128, 128, (M, K), generator=g, device="cuda").to(torch.int8)
        B = torch.randint(-128, 128, (N, K), generator=g, device="cuda").to(torch.int8)
        top = 127.0 * 127.0 / 3
    else:
        A = torch.randint(0, 256, (M, K // 2), generator=g, device="cuda").to(torch.uint8)
        B = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda").to(torch.uint8)
        top = 21.0
    rs = (torch.rand(M, generator=g, device="cuda") + 0.5) * 2.0 / math.sqrt(K * top * top)
    cs = torch.rand(N, generator=g, device="cuda") + 0.5
    return A, B, rs, cs


def call(prec, A, B, rs, cs, **kw):
    if prec == "fp16":
        return binding.gemm_fp16_linear(A, B, **kw)
    return (binding.gemm_s8_linear if prec == "s8" else binding.gemm_s4_linear)(A, B, rs, cs, **kw)


def check(prec, A, B, rs, cs, bias, act, residual, got):
    a, b = (A.double(), B.double()) if prec != "s4" else (unpack(A).double(), unpack(B).double())
    x = a @ b.t()
    if prec == "fp16":
        e = 1e-4 * (a.abs() @ b.abs().t()) + 1e-6
    else:
        x = x * rs.double()[:, None] * cs.double()
        e = 4 * U32 * x.abs()
    if bias is not None:
        x = x + bias.double()
        e = e + U32 * (x.abs() + bias.double().abs())
    y = activate(x, act)
    e = 1.13 * e + 1e-6 * x.abs()
    if residual is not None:
        y = y + residual.double()
        e = e + U32 * y.abs()
    if got.dtype == torch.float16:
        e = e + 2.0 ** -11 * y.abs() + 2.0 ** -25
    err = (got.double() - y).abs()       # (an exact zero has a bound of zero; a NaN fails)
    assert (err <= e).all(), "%.3g x bound" % (err / e.clamp(min=1e-30)).max().item()


def extras(M, N, dtype, seed, bias=True, residual=True):
    g = rng(seed + 1)
    return (torch.randn(N, generator=g, device="cuda") if bias else None,
            torch.randn(M, N, generator=g, device="cuda").to(dtype) if residual else None)


# every kernel: few rows on either side, exchanged operands, cluster split-K, one-CTA and pair tiles
SHAPES = [(1, 512, 64), (1, 4096, 4096), (7, 1000, 1056), (16, 2050, 512), (24, 1024, 2048), (33, 1111, 320),
          (64, 4096, 8192), (100, 3, 64), (1030, 5, 96), (130, 264, 4128), (333, 1001, 1088), (512, 512, 512),
          (700, 2048, 256), (2048, 1024, 1024)]


@pytest.mark.parametrize("prec", ["fp16", "s8", "s4"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_shapes(prec, M, N, K):
    A, B, rs, cs = operands(prec, M, N, K, M + N + K)
    for dtype in (torch.float16, torch.float32):
        bias, residual = extras(M, N, dtype, M)
        got = call(prec, A, B, rs, cs, bias=bias, activation="gelu_tanh", residual=residual, out_dtype=dtype)
        check(prec, A, B, rs, cs, bias, "gelu_tanh", residual, got)


@pytest.mark.parametrize("act", list(binding.ACTIVATIONS))
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("M,N", [(9, 777), (150, 136)])
def test_every_stage(act, bias, residual, M, N):
    for prec in ("fp16", "s8"):
        A, B, rs, cs = operands(prec, M, N, 256, 3)
        A = A * 4 if prec == "fp16" else A      # values up to +-20: both ends of the activations
        bi, re = extras(M, N, torch.float32, 4, bias, residual)
        got = call(prec, A, B, rs, cs, bias=bi, activation=act, residual=re, out_dtype=torch.float32)
        check(prec, A, B, rs, cs, bi, act, re, got)


@pytest.mark.parametrize("bn,cta_group", [(32, 1), (64, 1), (128, 1), (256, 1), (64, 2), (128, 2), (256, 2)])
@pytest.mark.parametrize("prec", ["fp16", "s8"])
def test_every_tile_shape(prec, bn, cta_group):
    M, N, K = 650, 1096, 1184
    A, B, rs, cs = operands(prec, M, N, K, bn)
    binding.gemm_set_config_override(bn, 0, cta_group)
    for dtype in (torch.float32,) if bn == 32 else (torch.float16, torch.float32):
        bias, residual = extras(M, N, dtype, 5)
        got = call(prec, A, B, rs, cs, bias=bias, activation="silu", residual=residual, out_dtype=dtype)
        check(prec, A, B, rs, cs, bias, "silu", residual, got)


@pytest.mark.parametrize("prec", ["fp16", "s8"])
@pytest.mark.parametrize("M,N", [(1100, 1208), (1100, 1207)])
def test_wide_kernel(prec, M, N):
    binding.gemm_set_kernel_family(2)
    A, B, rs, cs = operands(prec, M, N, 2048, 6)
    for dtype in (torch.float16, torch.float32):
        bias, residual = extras(M, N, dtype, 7)
        got = call(prec, A, B, rs, cs, bias=bias, activation="gelu", residual=residual, out_dtype=dtype)
        check(prec, A, B, rs, cs, bias, "gelu", residual, got)


@pytest.mark.parametrize("scheme", [1, 2, 5, 6])
@pytest.mark.parametrize("M,N,K", [(48, 1500, 2080), (600, 1100, 1056), (2048, 2048, 2048)])
def test_s4_routes(scheme, M, N, K):
    A, B, rs, cs = operands("s4", M, N, K, scheme)
    binding.gemm_set_s4_scheme(scheme)
    for dtype in (torch.float16, torch.float32):
        bias, residual = extras(M, N, dtype, 8)
        got = call("s4", A, B, rs, cs, bias=bias, activation="relu", residual=residual, out_dtype=dtype)
        check("s4", A, B, rs, cs, bias, "relu", residual, got)


@pytest.mark.parametrize("swap", [1, 2])
@pytest.mark.parametrize("M,N", [(60, 1300), (300, 520)])
def test_operand_order(swap, M, N):
    binding.gemm_set_swap_ab(swap)
    for prec in ("fp16", "s8"):
        A, B, rs, cs = operands(prec, M, N, 512, 11)
        for dtype in (torch.float16, torch.float32):
            bias, residual = extras(M, N, dtype, 12)
            got = call(prec, A, B, rs, cs, bias=bias, activation="silu", residual=residual, out_dtype=dtype)
            check(prec, A, B, rs, cs, bias, "silu", residual, got)


@pytest.mark.parametrize("M", [1, 5, 40, 300])
@pytest.mark.parametrize("offset,pitch", [(0, 2048), (8, 1300), (3, 1201)])
def test_pitches_and_in_place(M, offset, pitch):
    """C and residual as column blocks of larger matrices; nothing outside the block is touched."""
    N, K = 1100, 256
    for prec in ("fp16", "s8", "s4"):
        A, B, rs, cs = operands(prec, M, N, K, M)
        for dtype in (torch.float16, torch.float32):
            bias, _ = extras(M, N, dtype, 9)
            big = torch.randn(M, pitch, generator=rng(10), device="cuda").to(dtype)
            res = torch.randn(M, pitch + 5, generator=rng(13), device="cuda").to(dtype)[:, 2:2 + N]
            before = big.clone()
            got = call(prec, A, B, rs, cs, bias=bias, activation="silu", residual=res, C=big[:, offset:offset + N])
            check(prec, A, B, rs, cs, bias, "silu", res, got)
            assert torch.equal(big[:, :offset], before[:, :offset])
            assert torch.equal(big[:, offset + N:], before[:, offset + N:])


@pytest.mark.parametrize("M,N,K", [(4, 1024, 512), (48, 2048, 512), (300, 520, 320), (640, 768, 1024)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_residual_in_place(M, N, K, dtype):
    for prec in ("fp16", "s8", "s4"):
        A, B, rs, cs = operands(prec, M, N, K, M)
        bias, x = extras(M, N, dtype, 14)
        before = x.clone()
        got = call(prec, A, B, rs, cs, bias=bias, residual=x, C=x)
        assert got.data_ptr() == x.data_ptr()
        check(prec, A, B, rs, cs, bias, "none", before, x)


def test_not_a_number_stays_where_it_is():
    A, B, _, _ = operands("fp16", 40, 600, 256, 1)
    A[3, 17] = float("nan")
    for act in binding.ACTIVATIONS:
        out = binding.gemm_fp16_linear(A, B, activation=act)
        assert torch.isnan(out[3]).all() and torch.isfinite(out[:3]).all() and torch.isfinite(out[4:]).all()


def test_another_stream_and_a_chain():
    """Quantise, INT8 layer with activation, quantise, INT8 layer onto the residual stream."""
    stream = torch.cuda.Stream()
    M, K, F = 37, 512, 1536
    x = torch.randn(M, K, generator=rng(20), device="cuda").half()
    w1, w2 = operands("s8", F, F, K, 21)[1], operands("s8", K, K, F, 22)[1]
    c1 = torch.full((F,), 1e-3, device="cuda")
    c2 = torch.full((K,), 1e-3, device="cuda")
    torch.cuda.synchronize()
    q1, s1 = binding.gemm_quantize_rows(x, stream=stream)
    h = binding.gemm_s8_linear(q1, w1, s1, c1, activation="gelu", stream=stream)
    q2, s2 = binding.gemm_quantize_rows(h, stream=stream)
    y = binding.gemm_s8_linear(q2, w2, s2, c2, residual=x, stream=stream)
    stream.synchronize()
    check("s8", q1, w1, s1, c1, None, "gelu", None, h)
    check("s8", q2, w2, s2, c2, None, "none", x, y)


# ------------------------------------------------------------------------- row quantisation
@pytest.mark.parametrize("prec", ["s8", "s4"])
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 8192), (3, 64), (5, 2080), (64, 1024), (129, 1056), (1000, 4096),
                                    (2, 40000), (1, 131040)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_quantize_rows(prec, rows, K, dtype):
    """Codes and scales equal the definition's FP32 arithmetic bit for bit, and the value of a code is within
    half a step of the input."""
    top = 127.0 if prec == "s8" else 7.0
    x = (torch.randn(rows, K, generator=rng(rows + K), device="cuda") * 3).to(dtype)
    if rows > 2:
        x[1] = 0
        x[2] = torch.finfo(torch.float16).smallest_normal * 2.0 ** -10      # the least binary16 value
    q, s = binding.gemm_quantize_rows(x, prec)
    amax = x.float().abs().amax(1)
    top_t = torch.full_like(amax, top)     # (dividing by a Python number multiplies by its inverse)
    assert torch.equal(s, amax / top_t)
    inv = torch.where(amax > 0, top_t / amax, torch.zeros_like(amax))
    want = torch.round(x.float() * inv[:, None]).to(torch.int32)
    codes = q.to(torch.int32) if prec == "s8" else unpack(q).to(torch.int32)
    assert torch.equal(codes, want) and codes.abs().max() <= top
    off = (codes.double() * s.double()[:, None] - x.double()).abs()
    assert (off <= s.double()[:, None] * (0.5 + 4 * top * U32)).all()


@pytest.mark.parametrize("offset", [0, 1, 3, 8])
def test_quantize_rows_of_a_block(offset):
    for dtype in (torch.float16, torch.float32):
        x = torch.randn(33, 700, generator=rng(2), device="cuda").to(dtype)[:, offset:offset + 640]
        for prec in ("s8", "s4"):
            q, s = binding.gemm_quantize_rows(x, prec)
            q2, s2 = binding.gemm_quantize_rows(x.contiguous(), prec)
            assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_quantize_rows_not_finite(bad):
    x = torch.randn(6, 512, generator=rng(2), device="cuda").half()
    x[2, 100] = bad
    for prec in ("s8", "s4"):
        q, s = binding.gemm_quantize_rows(x, prec)
        assert not torch.isfinite(s[2]) and torch.isfinite(s[[0, 1, 3, 4, 5]]).all()
        w = operands(prec, 40, 40, 512, 3)[1]
        y = (binding.gemm_s8_linear if prec == "s8" else binding.gemm_s4_linear)(
            q, w, s, torch.ones(40, device="cuda"))
        assert torch.isnan(y[2]).all() and torch.isfinite(y[[0, 1, 3, 4, 5]]).all()


# Long sums, FP32 results: parts of 2048 products are 128 accumulations, each cutting off 0.72 units of 2^-24 of an
# accumulator that has on average 2/3 of its final size: 128 * 0.72 * 2/3 * 2^-24 = 3.7e-6 of the result's norm, plus
# the rounded sums of up to nine parts (1e-6).  (One chain over all of K = 16408 would leave 3e-5.)
@pytest.mark.parametrize("M,N,K", [(1, 640, 16400), (8, 4096, 8200), (40, 1000, 16384), (64, 512, 16408),
                                   (333, 1001, 4104), (300, 512, 2056), (652, 176, 12536), (2000, 2000, 16408),
                                   (2500, 4096, 6152), (4096, 4096, 4096)])
@pytest.mark.parametrize("cfg", [None, (64, 1), (128, 1), (256, 1), (256, 2)])
def test_long_sums_keep_fp32(M, N, K, cfg):
    A, B, _, _ = operands("fp16", M, N, K, K + N)
    bias = torch.randn(N, generator=rng(5), device="cuda")
    res = torch.randn(M, N, generator=rng(6), device="cuda")
    if cfg:
        binding.gemm_set_config_override(*cfg, 1)
    x = A.double() @ B.double().t()
    y = binding.gemm_fp16_linear(A, B, out_dtype=torch.float32)
    assert (y.double() - x).norm() <= 4.7e-6 * x.norm()
    z = binding.gemm_fp16_linear(A, B, bias, "gelu", res, out_dtype=torch.float32)
    want = activate(x + bias.double(), "gelu") + res.double()
    assert (z.double() - want).norm() <= 4.7e-6 * 1.13 * x.norm() + 2e-6 * want.norm()
