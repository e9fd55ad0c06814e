"""The 4-bit cache and prompt attention where sizes and sharing are unusual: caches of more than 2^31 bytes, pages that sequences
share, calls on two streams at once, bounds far above what is there, long prompts."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_attention_fp16 import make as make_prompt, reference as prompt_reference
from test_gpu_kv4_attention import reference, setup
from test_gpu_kv4_cache import held
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def test_cache_beyond_32_bits():
    """Pages at the end of arrays of 2.3 GB: byte and token offsets pass 2^31."""
    pages, page, dim, n = 560_000, 128, 64, 300
    cache = binding.kv_cache_u4(pages, 1, page, dim)
    table = dev([[pages - 1, 0, pages - 2]])
    x = torch.randn(n, 3, 1, dim, device="cuda").half()
    binding.kv_append_u4(cache, x[:, 0], x[:, 1], dev([0, n]), dev([0]), table, n)
    k, v = binding.kv_read_u4(cache, dev([0, n]), dev([0]), table, n, tokens=n)
    for got, want in ((k, x[:, 0]), (v, x[:, 1])):
        assert torch.equal(got.cpu(), torch.from_numpy(held(want.cpu().numpy())[0]))
    assert cache[0][pages - 2].any() and not cache[0][pages // 2].any()
    for last in (1, 40):                  # few rows, many rows
        q = x[-last:, 2].contiguous()
        got = binding.kv_attention_u4(q, cache, dev([0, last]), dev([n]), table, last)
        ref, tol = reference(q, cache, table.cpu().numpy(), [n], [last], 0, dim ** -0.5)
        assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("news", [[1, 1, 1], [20, 1, 33]])
def test_shared_pages(news):
    """Sequences with a common prefix in the same pages."""
    lens = [200, 180, 260]
    cache, table, q = setup(lens, news, 8, 2, 128, 32, seed=4)
    table[1, :4] = table[2, :4] = table[0, :4]
    got = binding.kv_attention_u4(q, cache, dev(starts(news)), dev(lens), dev(table), max(news))
    ref, tol = reference(q, cache, table, lens, news, 0, 128 ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("news", [1, 64])
def test_two_streams_at_once(news):
    """Scratch for joined parts is a stream's own."""
    runs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        cache, table, q = setup([9000 + 500 * i], [news], 8, 2, 128, 64, seed=20 + i)
        args = (q, cache, dev([0, news]), dev([9000 + 500 * i]), dev(table), news)
        runs.append((args, binding.kv_attention_u4(*args)))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i in range(2):
            outs[i].append(binding.kv_attention_u4(*runs[i][0], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, runs[i][1]) for o in outs[i])


def test_bounds_far_above_what_is_there():
    """max_q, max_len and tables sized for the largest batch that a program will ever have."""
    lens, news = [70, 3, 0, 400], [1, 2, 0, 5]
    cache, table, q = setup(lens, news, 8, 2, 128, 16, seed=5)
    wide = torch.full((4, 5000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = dev(table)
    want = binding.kv_attention_u4(q, cache, dev(starts(news)), dev(lens), dev(table), 5)
    ref, tol = reference(q, cache, table, lens, news, 0, 128 ** -0.5)
    got = binding.kv_attention_u4(q, cache, dev(starts(news)), dev(lens), wide, 2 ** 20)
    for o in (want, got):
        assert ((o.double() - ref).abs() <= tol).all()
    q, k, v = (t.contiguous() for t in make_prompt(90, 4, 2, 64))
    cu = dev([0, 50, 90])
    assert torch.equal(binding.attention_fp16(q, k, v, cu, 50), binding.attention_fp16(q, k, v, cu, 2 ** 30))


def test_single_tokens_beside_prompts():
    """One call with sequences for both kernels: each takes its own and leaves the other's rows alone."""
    lens, news = [900, 70, 500, 33, 1200], [300, 1, 2, 33, 1]
    cache, table, q = setup(lens, news, 4, 2, 128, 32, seed=6)
    got = binding.kv_attention_u4(q, cache, dev(starts(news)), dev(lens), dev(table), 300)
    ref, tol = reference(q, cache, table, lens, news, 0, 128 ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()


def test_long_prompt():
    q, k, v = make_prompt(20001, 2, 1, 64, seed=7)
    got = binding.attention_fp16(q, k, v, dev([0, 20001]), 20001)
    ref, tol = prompt_reference(q, k, v, [20001], True, 0, 64 ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()


def test_nothing_to_do():
    cache, table, q = setup([20], [1], 4, 2, 64, 16)
    e = q[:0]
    assert binding.kv_attention_u4(e, cache, dev([0, 0]), dev([20]), dev(table), 1).shape == e.shape
    binding.kv_append_u4(cache, e[:, :2], e[:, :2], dev([0, 0]), dev([0]), dev(table), 1)
    assert binding.kv_read_u4(cache, dev([0, 0]), dev([0]), dev(table), 1)[0].shape == (0, 2, 64)
    assert binding.attention_fp16(e, e[:, :2], e[:, :2], dev([0, 0]), 1).shape == e.shape
    assert binding.rotary_fp16(e, None, dev([]), torch.ones(32, device="cuda")).shape == e.shape
    with pytest.raises(binding.GemmError):
        binding.attention_fp16(q, q[:, :2], q[:, :2], dev([0]), 1)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4, 1000])
@pytest.mark.parametrize("news", [[8, 5, 2], [100, 70, 9]])
def test_wide_windows_over_short_sequences(news, window):
    """More queries than tokens: the first stand at positions below 0, from which a window may reach further down than 32 bits do."""
    lens = [4, 60, 1]
    cache, table, q = setup(lens, news, 4, 2, 64, 16, seed=8)
    got = binding.kv_attention_u4(q, cache, dev(starts(news)), dev(lens), dev(table), max(news), window=window)
    ref, tol = reference(q, cache, table, lens, news, window, 64 ** -0.5)
    assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("batch", [9, 64])
def test_sequences_that_overlap(batch):
    """Row counts that fall and rise again name more rows than there are: reported, and nothing is written outside the result."""
    rows = 1000
    cu = dev([0 if i % 2 == 0 else rows for i in range(batch + 1)])
    cache, table, q = setup([rows] * batch, [rows], 4, 2, 64, 16, seed=9)
    guarded = torch.zeros(rows + 256, 4, 64, device="cuda").half()
    binding.kv_attention_u4(q, cache, cu, dev([rows] * batch), dev(table), rows, out=guarded[128:128 + rows])
    assert binding.gemm_last_device_status() == 6
    binding.attention_fp16(q, q[:, :2], q[:, 2:], cu, rows, out=guarded[128:128 + rows])
    assert binding.gemm_last_device_status() == 6
    assert not guarded[:128].any() and not guarded[128 + rows:].any()
