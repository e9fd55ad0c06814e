"""INT8 key/value cache: writing and reading back against the definition.

The definition's arithmetic is FP32 with IEEE operations, so codes and scales are compared for
equality with the same operations in numpy, and the values with the 64-bit inputs: a code that was
never requantised is within half a step of its input."""
import numpy as np
import pytest
import torch

from paper_2608_10103_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def make_table(lens, page, extra=3, seed=0):
    """A block table of shuffled pages; entries past a sequence's length point nowhere."""
    pages = [-(-n // page) for n in lens]
    order = np.random.default_rng(seed).permutation(sum(pages) + extra)
    width = max(max(pages), 1) + 1
    table = np.full((len(lens), width), -7, dtype=np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(pages) + extra


class Model:
    """The definition, page by page, in FP32."""

    def __init__(self, pages, heads, page, dim):
        self.code = np.zeros((pages, heads, page, dim), dtype=np.float32)
        self.scale = np.zeros((pages, heads), dtype=np.float32)
        self.page = page

    def append(self, x, cu, past, table):
        f = np.float32
        for b in range(len(past)):
            n = cu[b + 1] - cu[b]
            if n == 0:
                continue
            for j in range(past[b] // self.page, (past[b] + n - 1) // self.page + 1):
                lo, hi = max(past[b], j * self.page), min(past[b] + n, (j + 1) * self.page)
                new = x[cu[b] + lo - past[b]: cu[b] + hi - past[b]].astype(f).transpose(1, 0, 2)
                slot, old = table[b, j], max(0, past[b] - j * self.page)
                was = self.scale[slot] if old else np.zeros_like(self.scale[slot])
                now = np.maximum(was, np.abs(new).max((1, 2)) / f(127))
                inv = np.where(now > 0, f(1) / np.where(now > 0, now, f(1)), f(0)).astype(f)
                self.code[slot][:, :old] = np.rint(self.code[slot][:, :old] * (was * inv)[:, None, None])
                self.code[slot][:, lo - j * self.page: hi - j * self.page] = np.rint(new * inv[:, None, None])
                self.scale[slot] = now

    def read(self, cu, first, table):
        rows = []
        for b in range(len(first)):
            for pos in range(first[b], first[b] + cu[b + 1] - cu[b]):
                slot = table[b, pos // self.page]
                rows.append(self.code[slot][:, pos % self.page] * self.scale[slot][:, None])
        shape = (0, self.code.shape[1], self.code.shape[3])
        return np.stack(rows).astype(np.float16) if rows else np.zeros(shape, np.float16)


def starts(counts):
    return [int(v) for v in np.concatenate(([0], np.cumsum(counts)))]


@pytest.mark.parametrize("page,heads,dim", [(16, 1, 64), (16, 8, 128), (32, 3, 256), (64, 8, 128), (128, 2, 64),
                                            (128, 5, 256)])
def test_append_and_read(page, heads, dim):
    """Prompts of several lengths, zero among them, then token after token, larger and larger."""
    g = np.random.default_rng(page + heads)
    steps = [[0, 1, page, 3 * page + 5, page - 1], [1, 1, 1, 1, 1], [0, 2, 5, 1, page + 3], [1, 1, 1, 1, 1],
             [1, 0, 1, 0, 1]]
    final = [sum(s[b] for s in steps) for b in range(5)]
    table, pages = make_table(final, page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    for t in cache[:2]:
        t.fill_(99)                 # what an earlier owner of the pages left
    for t in cache[2:]:
        t.fill_(1e4)
    models = (Model(pages, heads, page, dim), Model(pages, heads, page, dim))
    past = [0] * 5
    for i, new in enumerate(steps):
        cu = starts(new)
        rows = torch.from_numpy((g.standard_normal((cu[-1], 2, heads, dim)) * (1 + i)).astype(np.float16)).cuda()
        k, v = rows[:, 0], rows[:, 1]               # one buffer: a token stride of 2 heads dim
        binding.kv_append_s8(cache, k, v, dev(cu), dev(past), dev(table), max(new))
        for m, x in zip(models, (k, v)):
            m.append(x.cpu().numpy(), cu, past, table)
        past = [a + b for a, b in zip(past, new)]
        cu = starts(past)
        got = binding.kv_read_s8(cache, dev(cu), dev([0] * 5), dev(table), max(past))
        for m, t in zip(models, got):
            assert np.array_equal(t.cpu().numpy(), m.read(cu, [0] * 5, table))
    for m, codes, scale in zip(models, cache[:2], cache[2:]):
        for b in range(5):
            for j in range(-(-past[b] // page)):
                slot, n = table[b, j], min(page, past[b] - j * page)
                assert np.array_equal(codes[slot, :, :n].cpu().numpy(), m.code[slot][:, :n])
                assert np.array_equal(scale[slot].cpu().numpy(), m.scale[slot])
                assert (codes[slot, :, n:] == 99).all()        # positions without a token are left alone
    # part of the sequences, from the middle
    first, count = [0, 1, 2, page, page - 3], [1, 1, page, 7, 5]
    cu = starts(count)
    got = binding.kv_read_s8(cache, dev(cu), dev(first), dev(table), max(count), tokens=cu[-1])
    for m, t in zip(models, got):
        assert np.array_equal(t.cpu().numpy(), m.read(cu, first, table))


def test_values_are_within_half_a_step():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n, heads, dim, page = 300, 4, 128, 32
    x = (torch.randn(n, heads, dim, generator=g, device="cuda") * 5).half()
    table, pages = make_table([n], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    binding.kv_append_s8(cache, x, x, dev([0, n]), dev([0]), dev(table), n)
    for codes, scale in ((cache[0], cache[2]), (cache[1], cache[3])):
        slots = dev(table[0, :-(-n // page)]).long()
        value = (codes[slots].double() * scale[slots].double()[..., None, None]).transpose(1, 2).reshape(-1, heads, dim)[:n]
        step = scale[slots].double()[:, None, :].expand(-1, page, -1).reshape(-1, heads)[:n]
        assert ((value - x.double()).abs() <= step[..., None] * (0.5 + 127 * 2.0 ** -22)).all()


def test_zeros_and_values_that_are_not_finite():
    heads, dim, page = 2, 64, 16
    table, pages = make_table([40, 20], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    x = torch.zeros(60, heads, dim, device="cuda", dtype=torch.float16)
    x[40:] = 1.5
    x[45, 1, 3] = float("inf")
    y = x.clone()
    y[45, 1, 3] = float("nan")
    binding.kv_append_s8(cache, x, y, dev([0, 40, 60]), dev([0, 0]), dev(table), 40)
    for t in binding.kv_read_s8(cache, dev([0, 40, 60]), dev([0, 0]), dev(table), 40):
        assert (t[:40] == 0).all()
        assert not torch.isfinite(t[40:56, 1]).any()           # the poisoned page of that head
        assert torch.isfinite(t[40:56, 0]).all() and torch.isfinite(t[56:]).all()
    # a NaN stays in its page when more tokens follow; a page that starts afresh forgets it
    more = torch.ones(1, heads, dim, device="cuda", dtype=torch.float16)
    binding.kv_append_s8(cache, more, more, dev([0, 0, 1]), dev([40, 14]), dev(table), 1)
    k, _ = binding.kv_read_s8(cache, dev([0, 0, 15]), dev([0, 0]), dev(table), 15)
    assert not torch.isfinite(k[:, 1]).any()
    binding.kv_append_s8(cache, more, more, dev([0, 0, 1]), dev([40, 0]), dev(table), 1)
    k, _ = binding.kv_read_s8(cache, dev([0, 0, 1]), dev([0, 0]), dev(table), 1)
    assert torch.isfinite(k).all()


def test_offsets_beyond_32_bits():
    heads, dim, page = 16, 128, 128
    pages = 8300                                    # 2.2e9 codes each
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    table = np.array([[8299, 5, 8298]], dtype=np.int32)
    x = torch.randn(300, heads, dim, device="cuda").half()
    binding.kv_append_s8(cache, x, x, dev([0, 300]), dev([0]), dev(table), 300)
    k, v = binding.kv_read_s8(cache, dev([0, 300]), dev([0]), dev(table), 300)
    assert torch.equal(k, v)
    m = Model(3, heads, page, dim)
    m.append(x.cpu().numpy(), [0, 300], [0], np.array([[0, 1, 2]]))
    assert np.array_equal(k.cpu().numpy(), m.read([0, 300], [0], np.array([[0, 1, 2]])))


def test_bad_indices_are_reported_and_not_followed():
    heads, dim, page = 2, 64, 16
    cache = binding.kv_cache_s8(4, heads, page, dim)
    x = torch.ones(20, heads, dim, device="cuda", dtype=torch.float16)
    for table, past, cu, bound in (([[0, 4]], [0], [0, 20], 20), ([[0, -1]], [0], [0, 20], 20),
                                   ([[0, 1]], [20], [0, 20], 20), ([[0, 1]], [-1], [0, 20], 20),
                                   ([[0, 1]], [0], [0, 20], 10), ([[0, 1]], [0], [20, 0], 20)):
        binding.kv_append_s8(cache, x, x, dev(cu), dev(past), dev(table), bound)
        assert binding.gemm_last_device_status() == 6
        binding.kv_read_s8(cache, dev(cu), dev(past), dev(table), bound, tokens=20)
        assert binding.gemm_last_device_status() == 6
    assert (cache[0][2:] == 0).all() and (cache[2][2:] == 0).all()


def test_order_on_another_stream():
    stream = torch.cuda.Stream()
    heads, dim, page = 4, 128, 16
    table, pages = make_table([64], page)
    cache = binding.kv_cache_s8(pages, heads, page, dim)
    x = torch.randn(64, heads, dim, device="cuda").half()
    cu, past, tb = dev([0, 64]), dev([0]), dev(table)
    torch.cuda.synchronize()
    binding.kv_append_s8(cache, x, x, cu, past, tb, 64, stream=stream)
    k, v = binding.kv_read_s8(cache, cu, past, tb, 64, tokens=64, stream=stream)
    stream.synchronize()
    m = Model(pages, heads, page, dim)
    m.append(x.cpu().numpy(), [0, 64], [0], table)
    assert np.array_equal(k.cpu().numpy(), m.read([0, 64], [0], table)) and torch.equal(k, v)
