"""Attention over 4-bit values whose range does not contain zero: they are not rounded on their way into the product.

Queries are zero, so that every softmax weight is the same power of two, and the offsets of neighbouring tokens cancel: what is left is as
small as the codes' part, and a rounding of the values themselves would stand out. Tolerance per result, with A the largest |value| and n tokens:
binary16 result 2^-11 (2^-25); exponentials, factors and FP32 sums (2^-20 + n 2^-24) A; sums cut off 2e-9 n A; few rows: weights times the
value scale rounded to binary16, 2^-11 of 8 scale; many rows: what the first of two binary16 tiles leaves of a value, up to 2^-11 A and two scales, itself
rounded to binary16, 2^-11 of that."""
import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv4_attention import setup, values
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 12, 40, 200])
@pytest.mark.parametrize("far", [0.2, 1.0, 10.0, 100.0, 3000.0, 30000.0])
@pytest.mark.parametrize("size", [0.0667, 0.00021, 2.0 ** -17])
def test_values_far_from_zero(dim, rows, far, size):
    L, page = 520, 32
    cache, table, q = setup([L], [rows], 2, 2, dim, page, seed=rows)
    q.zero_()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    scale = (size * (1 + torch.rand(cache[3].shape[:3], generator=g, device="cuda"))).half()
    sign = 1.0 - 2.0 * (torch.arange(page, device="cuda") % 2)
    offset = (far * (1 + 0.01 * torch.rand(scale.shape, generator=g, device="cuda"))).half()
    offset[..., 1::2] = offset[..., 0::2]
    scale[..., 1::2] = scale[..., 0::2]
    cache[3][..., 0] = scale * sign          # pairs of tokens: one counts up from its offset, one down from minus that
    cache[3][..., 1] = offset * sign
    got = binding.kv_attention_u4(q, cache, dev([0, rows]), dev([L]), dev(table), rows)
    slots = dev(table[0, :-(-L // page)]).long()
    v = values(cache[1][slots], cache[3][slots])[0].transpose(0, 1).reshape(2, -1, dim)[:, :L]
    sums = torch.cumsum(v, dim=1)
    for i in range(rows):
        n = L - rows + i + 1
        ref = sums[:, n - 1] / n
        A, s = v.abs().max().item(), 2.0 * size
        tol = 2.0 ** -11 * ref.abs() + 2.0 ** -25 + (2.0 ** -20 + n * 2.0 ** -24 + 2e-9 * n) * A
        tol = tol + (2.0 ** -11 * 8 * s if rows <= 16 else 2.0 ** -11 * (2.0 ** -11 * A + 2 * s))
        err = (got[i].double() - ref).abs()
        assert (err <= tol).all(), (i, (err / tol).max().item())


@pytest.mark.parametrize("rows", [1, 40])
def test_one_token(rows):
    """A window of one: each result is the token's value, rounded once."""
    for dim in (64, 128, 256):
        cache, table, q = setup([200], [rows], 1, 1, dim, 16, seed=5)
        g = torch.Generator(device="cuda")
        g.manual_seed(4)
        cache[3][..., 1] = (cache[3][..., 1] + 100 * torch.randn(cache[3].shape[:3], generator=g, device="cuda")).half()
        got = binding.kv_attention_u4(q, cache, dev([0, rows]), dev([200]), dev(table), rows, window=1)
        slots = dev(table[0, :13]).long()
        v, top = (x.transpose(0, 1).reshape(1, -1, dim)[0, 200 - rows:200] for x in values(cache[1][slots], cache[3][slots]))
        tol = 2.0 ** -11 * v.abs() + 2.0 ** -25 + 2.0 ** -20 * top
        if rows <= 16:   # a weight times its scale in binary16, 2^-11 of up to 8 scale, against one in 32 bits
            tol = tol + 2.0 ** -11 * 8 * cache[3][slots][..., 0].abs().max().double()
        assert ((got[:, 0].double() - v).abs() <= tol).all()
