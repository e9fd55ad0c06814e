"""Rotary positions against the formula in 64 bits.

Tolerance per value: binary16 result 2^-11 of itself (2^-25 below its normal range); the angle to 5e-7
and FP32 products, 4 * 2^-24, of |x_a| + |x_b|."""
import pytest
import torch

from paper_2608_10103_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def reference(x, positions, inv_freq, sections, pairs):
    count = inv_freq.numel()
    axis = sum(([a] * n for a, n in enumerate(sections)), [])
    angle = positions.view(-1, x.shape[0])[axis].double().t() * inv_freq.double()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y, mag = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    i = torch.arange(count, device=x.device)
    first, second = (i, i + count) if pairs == "halves" else (2 * i, 2 * i + 1)
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    mag[..., first] = mag[..., second] = a.abs() + b.abs()
    return y, 2.0 ** -11 * y.abs() + 2.0 ** -25 + (5e-7 + 2.0 ** -22) * mag


def frequencies(rotary):
    return (10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float().cuda()


def make(tokens, heads, kv_heads, dim, axes, far, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows = torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g, device="cuda").half()
    pos = (torch.rand(axes, tokens, generator=g, device="cuda", dtype=torch.float64) * far).to(torch.int32)
    return rows[:, :heads], rows[:, heads:heads + kv_heads], pos


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,rotary,sections,far", [
    (1, 1, 1, 64, 64, (32,), 5), (1, 32, 8, 128, 128, (30, 17, 17), 32768), (333, 12, 2, 64, 48, (14, 10), 1000),
    (77, 3, 1, 256, 256, (64, 32, 16, 16), 1 << 22), (5000, 4, 4, 128, 112, (0, 56), 1 << 30), (129, 2, 1, 256, 16, (8,), 2 ** 31 - 1),
    (40, 5, 5, 72, 64, (11, 11, 10), 77), (9, 1, 3, 1024, 1024, (512,), 4096)])
def test_follows_the_formula(tokens, heads, kv_heads, dim, rotary, sections, far, pairs):
    q, k, pos = make(tokens, heads, kv_heads, dim, len(sections), far)
    pos[:, 0] = 0
    pos[-1, -1] = -far
    freq = frequencies(rotary)
    got = binding.rotary_fp16(q, k, pos, freq, sections, pairs)
    for x, y in zip((q, k), got):
        want, tol = reference(x, pos, freq, sections, pairs)
        assert y.is_contiguous() and ((y.double() - want).abs() <= tol).all()
        assert torch.equal(y[..., rotary:], x[..., rotary:])


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_in_place_out_and_without_keys(pairs):
    q, k, pos = make(70, 6, 2, 128, 3, 500, seed=1)
    freq, sections = frequencies(96), [20, 14, 14]
    want = binding.rotary_fp16(q, k, pos, freq, sections, pairs)
    base = q._base.clone() if q._base is not None else None
    only = binding.rotary_fp16(q, None, pos, freq, sections, pairs)
    assert torch.equal(only, want[0])
    out = torch.zeros(8, 70, 128, dtype=torch.float16, device="cuda").transpose(0, 1)   # heads in front of tokens
    binding.rotary_fp16(q, k, pos, freq, sections, pairs, out=(out[:, :6], out[:, 6:]))
    assert torch.equal(out[:, :6], want[0]) and torch.equal(out[:, 6:], want[1])
    r = binding.rotary_fp16(q, k, pos, freq, sections, pairs, out=(q, k))
    assert r[0] is q or r[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(q._base[:, 8:], base[:, 8:])     # the values beside them


def test_one_axis_and_infinities():
    q, k, pos = make(4, 2, 1, 64, 1, 50, seed=2)
    freq = frequencies(64)
    a = binding.rotary_fp16(q, k, pos[0].contiguous(), freq)
    b = binding.rotary_fp16(q, k, pos, freq, (32,))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    q[1, 0, 3] = float("inf")
    c = binding.rotary_fp16(q, k, pos, freq)[0]
    bad = ~torch.isfinite(c)
    want = torch.zeros_like(bad)
    want[1, 0, 3] = want[1, 0, 35] = True
    assert torch.equal(bad, want)


def test_other_stream_and_graph():
    q, k, pos = make(300, 8, 2, 128, 3, 900, seed=3)
    freq, sections = frequencies(128), (30, 17, 17)
    want = binding.rotary_fp16(q, k, pos, freq, sections)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = binding.rotary_fp16(q, k, pos, freq, sections, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = tuple(torch.empty_like(w) for w in want)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.rotary_fp16(q, k, pos, freq, sections, out=out)
    pos += 11
    want = binding.rotary_fp16(q, k, pos, freq, sections)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_refusals():
    q, k, pos = make(8, 4, 2, 64, 2, 10)
    freq = frequencies(64)
    for bad in ((3, 30), (16, 16, 0), None, (40, -8)):
        with pytest.raises((ValueError, binding.GemmError)):
            binding.rotary_fp16(q, k, pos, freq, bad)
    for x in (q.float(), q[0], q.transpose(1, 2)):
        with pytest.raises((TypeError, ValueError)):
            binding.rotary_fp16(x, k, pos, freq, (16, 16))
    with pytest.raises(ValueError):
        binding.rotary_fp16(q, k[:4], pos, freq, (16, 16))
    with pytest.raises(ValueError):
        binding.rotary_fp16(q, k, pos[:, :4].contiguous(), freq, (16, 16))
    with pytest.raises(binding.GemmError):
        binding.rotary_fp16(q, k, pos, frequencies(64)[:20].contiguous(), (10, 10))   # 40 is no multiple of 16
    with pytest.raises(TypeError):
        binding.rotary_fp16(q, k, pos, freq, (16, 16), out=(q,))
    with pytest.raises(binding.GemmError):
        binding.rotary_fp16(q, k, pos, freq, (16, 16), out=(q[:1].expand(8, -1, -1), k))
