"""Weights far below the largest one: long flat tails behind a dominant token, and value scales of very different
size.

Bound per output, p the softmax weights of the 64-bit reference, s the value scales, n tokens: a weight is held in
binary16 with 2^7 or more for the largest p s seen, so it is off by 2^-11 of itself, below the type's normal range by
2^-25, i.e. 2^-32 of the largest p s times a code of at most 127; an FP32 score by 2^-20 of c sum |q k|, q by
max|q| / (127 * 508) a value (few rows only), both in numerator and denominator; binary16 result 2^-11 (2^-25)."""
import math

import pytest
import torch

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import setup
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


def reference(q, cache, table, lens, news, scale, few_rows):
    k, v, ks, vs = cache
    heads, page, dim = k.shape[1:]
    out, tol, rels, at = [], [], [], 0
    for b, (L, n) in enumerate(zip(lens, news)):
        x = q[at:at + n].double().view(n, heads, -1, dim)
        at += n
        slots = dev(table[b, :-(-L // page)]).long()

        def rows(codes, s):
            return (codes[slots].double() * s[slots].double()[..., None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, :L]

        kk, vv = rows(k, ks), rows(v, vs)
        step = vs[slots].double()[..., None].expand(-1, -1, page).transpose(0, 1).reshape(heads, -1)[:, :L]
        sc = torch.einsum("nhgd,htd->nhgt", x, kk) * scale
        mag = torch.einsum("nhgd,htd->nhgt", x.abs(), kk.abs()).amax(3, keepdim=True) * scale
        hidden = torch.arange(L, device="cuda")[None] > L - n + torch.arange(n, device="cuda")[:, None]
        w = sc.masked_fill(hidden[:, None, None, :], -math.inf).softmax(3)
        o = torch.einsum("nhgt,htd->nhgd", w, vv)
        mass = torch.einsum("nhgt,htd->nhgd", w, vv.abs())
        rel = 2.0 ** -11 + 2 * 2.0 ** -20 * mag + 4e-6
        if few_rows:
            rel = rel + 2 * x.abs().amax(3, keepdim=True) * kk.abs().sum(2).amax(1)[None, :, None, None] * (scale / (127 * 508))
        floor = L * 2.0 ** -32 * 127 * (w * step[None, :, None]).amax(3, keepdim=True)
        out.append(o.reshape(n, -1, dim))
        tol.append((rel * mass + floor + 2.0 ** -11 * o.abs() + 2.0 ** -25).reshape(n, -1, dim))
        rels.append(float(rel.max()))
    return torch.cat(out), torch.cat(tol), max(rels)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("below", [16.3, 20.4, 25.2])
@pytest.mark.parametrize("new", [1, 64])
def test_flat_tail_behind_a_dominant_token(new, below, dim):
    """The first token outweighs each of the others by 2^below; its value is zero, so the result is the tail's."""
    batch, heads, length, page = 64 if new == 1 else 8, 8, 4096, 64
    cache, table, q = setup([length] * batch, [new] * batch, 4 * heads, heads, dim, page, spread=0.0)
    k, v, ks, vs = cache
    k.zero_()
    v.fill_(100)
    q.zero_()
    scale = dim ** -0.5
    q[..., 3] = 4.0
    ks.fill_(below * math.log(2) / (4.0 * 127 * scale))
    vs.fill_(0.5)
    for b in range(batch):
        k[int(table[b, 0]), :, 0, 3] = 127
        v[int(table[b, 0]), :, 0] = 0
    cu = dev([new * i for i in range(batch + 1)])
    got = binding.kv_attention_s8(q, cache, cu, dev([length] * batch), dev(table), new)
    ref, tol, rel = reference(q, cache, table, [length] * batch, [new] * batch, scale, new == 1)
    assert rel < 0.01 and (tol < 0.05 * ref).all()
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol).max().item()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,news", [([600, 1200], [1, 2]), ([600, 1200], [40, 64]), ([3000], [300])])
def test_value_scales_of_very_different_size(lens, news, dim):
    """Factors of e^4 a standard deviation between pages, in the values alone."""
    cache, table, q = setup(lens, news, 8, 2, dim, 16, spread=4.0, seed=6)
    cache[2].fill_(0.02)
    cu = dev([0] + list(torch.tensor(news).cumsum(0)))
    cache[3].clamp_(max=2.0)           # results stay inside binary16
    got = binding.kv_attention_s8(q, cache, cu, dev(lens), dev(table), max(news))
    few = max(news) * 4 <= (16 if dim == 256 else 32)
    ref, tol, rel = reference(q, cache, table, lens, news, dim ** -0.5, few)
    assert rel < 0.01
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g x bound" % (err / tol).max().item()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("tiny", [0.0, 1e-38, 2.0 ** -60, 1e-12])
def test_pages_of_no_size_beside_others(new, tiny):
    """Value scales that vanish: such pages come first, alone, then beside others; their tokens count all the same."""
    dim, page = 128, 16
    for lens in ([200], [2000]):
        cache, table, q = setup(lens, [new], 8, 2, dim, page, spread=0.0, seed=9)
        for part in (slice(0, -(-lens[0] // page)), slice(0, 8), slice(5, 7)):
            c = [t.clone() for t in cache]
            c[3][dev(table[0, part]).long()] = tiny
            got = binding.kv_attention_s8(q, c, dev([0, new]), dev(lens), dev(table), new)
            ref, tol, rel = reference(q, c, table, lens, [new], dim ** -0.5, new == 1)
            err = (got.double() - ref).abs()
            assert rel < 0.01 and (err <= tol).all(), "worst %.3g x bound" % (err / tol).max().item()
