"""A 4-bit cache that somebody else filled: scales of either sign, as a quantiser that counts from the maximum leaves them.

The value of a code is offset + code * scale whatever the sign; bounds are those of test_gpu_kv4_attention.py, which count with |scale|."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv4_attention import reference, setup
from test_gpu_kv_cache import dev, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def check(cache, table, q, lens, news, window=0):
    args = (dev(starts(news)), dev(lens), dev(table), max(news))
    got = binding.kv_attention_u4(q, cache, *args, window=window)
    ref, tol = reference(q, cache, table, lens, news, window, q.shape[2] ** -0.5)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol.clamp(min=1e-30)).max().item()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 4, 8, 9, 16, 17, 130])
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_negative_scales(dim, rows, which):
    """One token in two counts down from its maximum; and all of them."""
    lens, news = [90, 700, 2000 + rows], [min(rows, 90), rows, rows]
    for share in (0.5, 1.0):
        cache, table, q = setup(lens, news, 2, 2, dim, 32, seed=rows)
        g = torch.Generator(device="cuda")
        g.manual_seed(7)
        for i, name in ((2, "k"), (3, "v")):
            if which not in (name, "both"):
                continue
            turn = torch.rand(cache[i].shape[:3], generator=g, device="cuda") < share
            cache[i][..., 1] += torch.where(turn, 15 * cache[i][..., 0], 0)   # (rounded: a value of its own)
            cache[i][..., 0] *= torch.where(turn, -1, 1)
        check(cache, table, q, lens, news)
        check(cache, table, q, lens, news, window=100)


@pytest.mark.parametrize("news", [1, 40])
def test_counting_from_either_end_is_the_same(news):
    """offset + c scale = (offset + 15 scale) + (15 - c) (-scale): exact in binary16 with these numbers."""
    for dim in (64, 128, 256):
        cache, table, q = setup([500], [news], 4, 1, dim, 16, seed=news)
        for i in (2, 3):
            cache[i][..., 0], cache[i][..., 1] = 0.125, -1.0
        down = [255 - cache[0], 255 - cache[1], cache[2].clone(), cache[3].clone()]
        for i in (2, 3):
            down[i][..., 0], down[i][..., 1] = -0.125, 0.875
        args = (dev([0, news]), dev([500]), dev(table), news)
        a, b = binding.kv_attention_u4(q, cache, *args), binding.kv_attention_u4(q, tuple(down), *args)
        read = [binding.kv_read_u4(c, dev([0, 500]), dev([0]), dev(table), 500) for c in (cache, tuple(down))]
        assert torch.equal(read[0][0], read[1][0]) and torch.equal(read[0][1], read[1][1])
        # weights 2^-11, results 2^-11, each side; scores FP32
        assert ((a.float() - b.float()).abs() <= 2.0 ** -9 * 1.0).all()
