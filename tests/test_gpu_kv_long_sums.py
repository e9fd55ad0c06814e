"""Prompt chunks over long sequences: what the tensor core's accumulator cuts off must not add up over the tokens.

An accumulation of 16 tokens cuts off up to two units of 2^-24 of what is there, which on average is at most 2/3 of the end,
all with one sign.  A sum of 16384 tokens thus shrinks the result by up to 16384 / 16 * 2 * 2/3 * 2^-24 = 8e-5; the
other roundings have no sign (3e-4 a value, 1e-6 over the 9e4 values of a head).  The values themselves are held
against the definition in 64 bits with the bound of the attention tests."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def run(length, new, kv_heads, group, dim, mean=0.0, slope=0.0, window=0, page=64):
    g = torch.Generator(device="cuda")
    g.manual_seed(length + dim)
    pages = -(-length // page)
    cache = [(torch.randn(pages, kv_heads, page, dim, generator=g, device="cuda") * 36 + 36 * m).round().clamp(-127, 127).to(torch.int8)
             for m in (0.0, mean)] + [0.02 + 0.02 * torch.rand(pages, kv_heads, generator=g, device="cuda") for _ in range(2)]
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    if slope:        # scores grow along the sequence, so that sums made earlier are scaled down later
        cache[2][table[0].long()] *= torch.linspace(0.1, slope, pages, device="cuda")[:, None]
    q = torch.randn(new, kv_heads * group, dim, generator=g, device="cuda").half()
    got = binding.kv_attention_s8(q, tuple(cache), dev([0, new]), dev([length]), table, new, window=window)
    again = binding.kv_attention_s8(q, tuple(cache), dev([0, new]), dev([length]), table, new, window=window)
    assert torch.equal(got, again)
    for head in (0, kv_heads - 1):
        part = [c[:, head:head + 1].contiguous() for c in cache]
        mine = slice(head * group, head * group + group)
        ref, tol = reference(q[:, mine], part, table.cpu().numpy(), [length], [new], window, dim ** -0.5)
        yield got[:, mine].double(), ref, tol


@pytest.mark.parametrize("mean", [0.0, 0.3])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_no_shrinking(mean, dim):
    for got, ref, tol in run(131072, 700, 32 if dim < 256 else 16, 1, dim, mean=mean):
        assert ((got - ref).abs() <= tol).all()
        assert abs((((got - ref) * ref).sum() / (ref * ref).sum()).item()) <= 8e-5 + 3e-6


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("length,new,kv_heads,window", [(16384 + 300, 300, 80, 0), (16385, 290, 80, 0), (32769, 280, 80, 0),
                                                        (70000, 300, 32, 0), (131072, 190, 16, 0), (70000, 300, 80, 40000)])
def test_sums_in_scratch(length, new, kv_heads, window, dim):
    """Lengths around a sum's end, scores that grow along the sequence, tokens divided over CTAs, a window."""
    group = 1 if kv_heads == 80 else 4
    for got, ref, tol in run(length, new, kv_heads, group, dim, slope=3.0, window=window):
        assert ((got - ref).abs() <= tol).all()


def test_captured_into_a_graph():
    """The scratch of both kernels exists after one call of the same size; lengths are read when the graph runs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    page, pages, heads, dim, new = 64, 600, 40, 64, 300
    cache = tuple([torch.randint(-100, 100, (pages, heads, page, dim), generator=g, device="cuda").to(torch.int8) for _ in range(2)] +
                  [0.02 + 0.02 * torch.rand(pages, heads, generator=g, device="cuda") for _ in range(2)])
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    q = torch.randn(new, heads * 2, dim, generator=g, device="cuda").half()
    cu, lens, out = dev([0, new]), dev([pages * page]), torch.empty_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        binding.kv_attention_s8(q, cache, cu, lens, table, new, out=out)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.kv_attention_s8(q, cache, cu, lens, table, new, out=out)
    for length in (pages * page, 20000, 700, pages * page):
        lens.fill_(length)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want = binding.kv_attention_s8(q, cache, cu, lens, table, new)
        assert torch.equal(out, want)
