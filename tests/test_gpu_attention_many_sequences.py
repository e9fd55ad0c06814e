"""Attention of very many short sequences in one call: the time goes by their number, not by its square."""
import numpy as np
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_attention_fp16 import make, reference
from test_gpu_kv4_attention import check as check4
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def run(lens, q, k, v):
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    cu = dev(starts(lens))
    binding.attention_fp16(q, k, v, cu, max(lens))
    begin.record()
    got = binding.attention_fp16(q, k, v, cu, max(lens))
    end.record()
    torch.cuda.synchronize()
    return got, begin.elapsed_time(end)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 1000, 3000])
def test_every_sequence_is_found(n):
    """Sequences of all lengths, with and without rows, in no order: each gives what it gives alone."""
    g = np.random.default_rng(n)
    lens = [int(x) for x in g.choice([0, 0, 1, 3, 60, 64, 65, 130, 300], n)]
    lens[n // 2] = 700
    q, k, v = make(sum(lens), 4, 2, 64, seed=n)
    got, _ = run(lens, q, k, v)
    at = starts(lens)
    for i in sorted(set(g.integers(0, n, 40)) | {n // 2, n - 1}):
        if lens[i]:
            rows = slice(at[i], at[i + 1])
            alone = binding.attention_fp16(q[rows], k[rows], v[rows], dev([0, lens[i]]), lens[i])
            assert torch.equal(got[rows], alone)
    picked = [i for i in range(n) if lens[i] and i % 50 == 0]
    rows = torch.cat([torch.arange(at[i], at[i + 1]) for i in picked] + [torch.zeros(0, dtype=torch.int64)]).cuda()
    if len(rows):
        ref, tol = reference(q[rows], k[rows], v[rows], [lens[i] for i in picked], True, 0, 64 ** -0.5)
        assert ((got[rows].double() - ref).abs() <= tol).all()


def test_time_goes_by_the_number():
    times = []
    for n in (4096, 16384, 65536):
        q, k, v = make(3 * n, 2, 1, 64, seed=1)
        times.append(run([3] * n, q, k, v)[1])
    # (four times as many took sixteen times as long, 84 ms for the second)
    assert times[2] <= 8 * times[1] and times[1] <= 20.0, times


def test_many_chunks_over_the_cache():
    g = np.random.default_rng(3)
    news = [int(x) for x in g.choice([0, 1, 5, 17, 40], 700)]
    lens = [n + int(x) for n, x in zip(news, g.integers(0, 200, 700))]
    check4(lens, news, 4, 1, 64, 16)
    check4(lens, news, 20, 1, 128, 32, window=40)
