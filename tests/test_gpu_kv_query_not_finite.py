"""Queries that hold a NaN or an infinity: NaN where they see a token, zeros where they see none."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import reference, setup
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("length,new", [(2, 4), (0, 4), (30, 60), (0, 60), (5000, 40)])
def test_rows_that_see_nothing_are_zeros(length, new, dim, value):
    cache, table, q = setup([length], [new], 4, 1, dim, 16)
    ref, tol = reference(q, cache, table, [length], [new], 0, dim ** -0.5)
    q[::2, 1, 7] = value                       # every second query, one head
    got = binding.kv_attention_s8(q, cache, dev([0, new]), dev([length]), dev(table), new)
    nothing = torch.arange(new, device="cuda") < new - length
    assert (got[nothing] == 0).all()
    bad = torch.zeros(new, 4, dtype=torch.bool, device="cuda")
    bad[::2, 1] = True
    assert torch.isnan(got[bad & ~nothing[:, None]]).all()
    assert ((got.double() - ref).abs() <= tol)[~bad].all()


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [2, 60])
def test_every_score_infinite(new, dim, value):
    """Keys of one sign in the query's infinite channel: all scores are +inf, or all -inf, and 0 / 0 either way."""
    cache, table, q = setup([200], [new], 4, 1, dim, 16)
    cache[0][..., 7] = 5
    q[:, 2, 7] = value
    got = binding.kv_attention_s8(q, cache, dev([0, new]), dev([200]), dev(table), new)
    assert torch.isnan(got[:, 2]).all() and torch.isfinite(got[:, [0, 1, 3]]).all()
