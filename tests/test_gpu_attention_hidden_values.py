"""Prompt attention beside values that are not finite: what a query does not see leaves its result as it is, bit for bit, in prompts
of any length and in a time that does not grow with them; what it sees counts as the formula has it.

A hidden value's weight is 0 and its product with any finite value 0, so results beside hidden values are compared for equality with
those of finite ones."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_attention_fp16 import make
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def same(a, b):
    return a.contiguous().view(torch.int16) == b.contiguous().view(torch.int16)


def sees(lens, causal, window):
    """[row, token] of the packed arrays."""
    n = sum(lens)
    at = torch.arange(n, device="cuda")
    seq = torch.cat([torch.full((x,), i, device="cuda") for i, x in enumerate(lens)])
    m = seq[:, None] == seq[None]
    if causal:
        m &= at[None] <= at[:, None]
    if window:
        m &= at[None] > at[:, None] - window
    return m


def check(lens, q_heads, kv_heads, dim, bad, causal=True, window=0, behind=0):
    """bad: (token, KV head, d, value) of V."""
    n = sum(lens)
    q, k, v = (t.contiguous() for t in make(n + behind, q_heads, kv_heads, dim, seed=len(lens) + window))
    cu = dev(starts(lens))
    clean = v.clone()
    for t, h, d, _ in bad:
        clean[t, h, d] = 0
    want = binding.attention_fp16(q, k, clean, cu, max(lens), causal=causal, window=window)[:n]
    for t, h, d, x in bad:
        v[t, h, d] = x
    if behind:
        v[n:] = NAN
        k[n:] = NAN
    got = binding.attention_fp16(q, k, v, cu, max(lens), causal=causal, window=window)[:n]
    group, m = q_heads // kv_heads, sees(lens, causal, window)
    add = torch.zeros(n, q_heads, dim, device="cuda")
    for t, h, d, x in bad:
        if t < n:
            add[:, h * group:(h + 1) * group, d] += torch.where(m[:, t], x, 0.0)[:, None]
    expect = torch.where(add == 0, want.float(), add)
    assert (same(got, expect.half()) | (torch.isnan(got) & torch.isnan(expect))).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads", [(2, 2), (8, 2), (6, 2), (24, 1)])
def test_hidden_and_visible(dim, q_heads, kv_heads):
    h = kv_heads - 1
    for lens in ([300, 90], [64, 1, 129, 77]):
        n = sum(lens)
        for window in (0, 1, 40, 70):
            bad = [(n // 2, h, 3, NAN), (n // 3, 0, dim - 1, INF), (n - 1, h, 8, -INF), (lens[0], 0, 0, NAN)]
            check(lens, q_heads, kv_heads, dim, bad, window=window)
        check(lens, q_heads, kv_heads, dim, bad, causal=False)
        check(lens, q_heads, kv_heads, dim, bad, causal=False, behind=40)
        check(lens, q_heads, kv_heads, dim, bad, behind=200)


def test_infinities_add_up():
    """Of one sign they stay, of two they are a NaN, for the rows that see both."""
    bad = [(70, 0, 5, INF), (90, 0, 5, INF), (100, 0, 6, INF), (101, 0, 6, -INF), (102, 0, 7, -INF), (102, 0, 8, NAN), (103, 0, 8, INF)]
    for dim in (64, 128, 256):
        check([200], 4, 1, dim, bad)
        check([200], 4, 1, dim, bad, window=33)


def test_every_value():
    for dim in (64, 128, 256):
        for n, window in ((700, 0), (700, 100), (40, 0)):
            q, k, v = (t.contiguous() for t in make(n, 4, 2, dim, seed=1))
            for x in (NAN, INF):
                v.fill_(x)
                got = binding.attention_fp16(q, k, v, dev([0, n]), n, window=window)
                # (an infinity with a weight that rounds to nothing may be a NaN)
                assert (torch.isnan(got) if x != x else ~torch.isfinite(got)).all()


def test_score_of_minus_infinity_times_infinity():
    """exp(-inf) = 0 and 0 x inf is a NaN, also where another row of the tile hides the token."""
    q, k, v = (t.contiguous() for t in make(100, 2, 1, 64, seed=2))
    q[..., 0] = 1.0
    k[50, 0, 0] = -INF
    want = binding.attention_fp16(q, k, v, dev([0, 100]), 100)
    v[50, 0, 9] = INF
    got = binding.attention_fp16(q, k, v, dev([0, 100]), 100)
    assert torch.isfinite(want).all() and torch.isnan(got[50:, :, 9]).all()
    got[50:, :, 9] = want[50:, :, 9]
    assert same(got, want).all()


def timed(*a, **kw):
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    out = binding.attention_fp16(*a, **kw)
    end.record()
    torch.cuda.synchronize()
    return out, begin.elapsed_time(end)


@pytest.mark.parametrize("n,dim", [(300001, 64), (200001, 128), (150001, 256)])
@pytest.mark.parametrize("window", [0, 30000])
def test_long_prompts(n, dim, window):
    """A NaN in the last token, which a row tile's other rows do not see, and one in the middle."""
    q, k, v = (t.contiguous() for t in make(n + 50, 4, 1, dim, seed=3))
    cu, spots = dev([0, n]), (n - 1, n // 2 + 5)
    v[spots[0]] = v[spots[1]] = 0
    timed(q, k, v, cu, n, window=window)
    want, fast = timed(q, k, v, cu, n, window=window)
    v[n:] = NAN
    v[spots[0], 0, 2] = NAN
    v[spots[1], 0, 7] = INF
    got, slow = timed(q, k, v, cu, n, window=window)
    at = torch.arange(n, device="cuda")
    for t, d, x in ((spots[0], 2, NAN), (spots[1], 7, INF)):
        seen = at >= t
        if window:
            seen &= at < t + window
        assert (~torch.isfinite(got[:n][seen][..., d])).all()
        got[:n, :, d] = torch.where(seen[:, None], want[:n, :, d], got[:n, :, d])
    assert same(got[:n], want[:n]).all()
    # (rows one by one took seconds here; a row tile with such values takes a millisecond more)
    assert slow < 2 * fast + 20.0, (slow, fast)
