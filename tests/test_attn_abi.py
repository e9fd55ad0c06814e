"""CPU-only checks of the rotary, prompt-attention and 4-bit cache entry points: exports and refusals."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_10103_b200 import binding, build as lib_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


def test_header_and_binding_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "b200attn.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\bint ([a-z0-9_]+)\s*\(", text)))
    assert names == sorted(binding.ATTN_EXPORTS)
    for name in names:
        assert getattr(lib, name) is not None


def rows(**kw):
    d = dict(x=16, y=32, heads=2, x_token_stride=128, x_head_stride=64, y_token_stride=128, y_head_stride=64)
    d.update(kw)
    return ctypes.byref(binding._RotaryRows(**d))


def test_rotary_refusals(lib):
    def call(tokens=4, dim=64, rotary=64, pairs=0, q=rows(), k=rows(), pos=16, axes=2, stride=4, sections=(20, 12), freq=16):
        s = None if sections is None else (ctypes.c_int * len(sections))(*sections)
        return lib.rotary_fp16(tokens, dim, rotary, pairs, q, k, pos, axes, stride, s, freq, None)

    for kw in (dict(tokens=0), dict(dim=0), dict(dim=2048), dict(rotary=0), dict(rotary=80), dict(pairs=2), dict(q=None, k=None),
               dict(pos=None), dict(freq=None), dict(axes=0), dict(axes=5), dict(stride=3), dict(sections=None),
               dict(sections=(20, 13)), dict(sections=(20, 11)), dict(sections=(-1, 33)), dict(sections=(2 ** 31 - 1, 33)),
               dict(q=rows(x=None)), dict(q=rows(heads=0)), dict(k=rows(x_head_stride=32)), dict(k=rows(y_head_stride=32)),
               dict(q=rows(x_token_stride=-8)), dict(q=rows(y_token_stride=0)), dict(q=rows(y=16, y_token_stride=256))):
        assert call(**kw) == -1, kw
    for kw in (dict(dim=68), dict(rotary=24, sections=(6, 6)), dict(pos=18), dict(freq=18), dict(q=rows(x=24)), dict(k=rows(y=24)),
               dict(q=rows(x_token_stride=132)), dict(q=rows(y_head_stride=68))):
        assert call(**kw) == -2, kw
    assert call(q=rows(heads=1 << 21)) == -7
    assert call(tokens=2 ** 31 - 1, axes=1, sections=None) == -7


def test_prompt_attention_refusals(lib):
    def call(batch=1, cu=16, most=8, rows=8, hq=4, hk=2, dim=64, q=16, qt=256, qh=64, k=16, v=16, kt=128, kh=64, scale=0.1, causal=1,
             window=0, out=16, ot=256):
        return lib.attention_fp16(batch, cu, most, rows, hq, hk, dim, q, qt, qh, k, v, kt, kh, scale, causal, window, out, ot, None)

    for kw in (dict(batch=0), dict(cu=None), dict(most=0), dict(rows=0), dict(hq=0), dict(hk=0), dict(hq=3), dict(dim=32), dict(dim=96),
               dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(causal=2), dict(window=-1), dict(causal=0, window=4),
               dict(qh=32), dict(kh=32), dict(qt=0), dict(kt=0), dict(ot=128), dict(scale=0.0), dict(scale=float("nan")),
               dict(scale=float("inf"))):
        assert call(**kw) == -1, kw
    for kw in (dict(cu=18), dict(q=24), dict(k=24), dict(v=24), dict(out=24), dict(qt=260), dict(qh=68), dict(kt=132), dict(kh=68),
               dict(ot=260)):
        assert call(**kw) == -2, kw
    for kw in (dict(hq=258, ot=1 << 20), dict(hk=65536, hq=65536, ot=1 << 30), dict(rows=2 ** 31 - 1), dict(qt=1 << 40), dict(kh=1 << 40)):
        assert call(**kw) == -7, kw


def cache(**kw):
    d = dict(k=16, v=16, k_scale=16, v_scale=16, num_pages=4, kv_heads=2, page_size=16, head_dim=64)
    d.update(kw)
    return ctypes.byref(binding._KvCache(**d))


def test_kv_refusals(lib):
    def append(c, batch=1, cu=16, past=16, table=16, stride=4, most=8, k=16, v=16, ts=128, hs=64, rows=8):
        return lib.kv_append_u4(c, batch, cu, past, table, stride, most, k, v, ts, hs, rows, None)

    def read(c, batch=1, cu=16, first=16, table=16, stride=4, most=8, k=16, v=16, rows=8):
        return lib.kv_read_u4(c, batch, cu, first, table, stride, most, k, v, rows, None)

    def attend(c, batch=1, cu=16, lens=16, table=16, stride=4, most=1, heads=4, q=16, ts=256, hs=64, scale=0.1,
               window=0, out=16, os=256, rows=8):
        return lib.kv_attention_u4(c, batch, cu, lens, table, stride, most, heads, q, ts, hs, scale, window, out,
                                   os, rows, None)

    for f in (append, read, attend):
        assert f(None) == -1
        for kw in (dict(k=None), dict(v_scale=None), dict(num_pages=0), dict(kv_heads=0), dict(page_size=8),
                   dict(page_size=48), dict(page_size=256), dict(head_dim=32), dict(head_dim=96)):
            assert f(cache(**kw)) == -1, kw
        assert f(cache(k=24)) == -2 and f(cache(k_scale=20)) == -2 and f(cache(v_scale=24)) == -2
        assert f(cache(), batch=0) == -1 and f(cache(), cu=None) == -1 and f(cache(), table=None) == -1
        assert f(cache(), stride=0) == -1 and f(cache(), most=0) == -1 and f(cache(), rows=0) == -1
        assert f(cache(), cu=18) == -2 and f(cache(), table=18) == -2
    assert append(cache(), k=None) == -1 and append(cache(), hs=32) == -1
    assert append(cache(), k=24) == -2 and append(cache(), ts=130) == -2
    assert append(cache(), batch=1 << 30, most=64, rows=64) == -7 and read(cache(), batch=1 << 30, most=64, rows=64) == -7
    assert read(cache(), k=None, v=None) == -1 and read(cache(), k=24) == -2
    assert attend(cache(), heads=3) == -1 and attend(cache(), heads=0) == -1 and attend(cache(), window=-1) == -1
    assert attend(cache(), scale=0.0) == -1 and attend(cache(), scale=float("nan")) == -1
    assert attend(cache(), out=None) == -1 and attend(cache(), os=128) == -1 and attend(cache(), ts=0) == -1
    assert attend(cache(), q=24) == -2 and attend(cache(), hs=68) == -2
    assert attend(cache(), heads=258, os=1 << 20) == -7 and attend(cache(), ts=1 << 40) == -7


def test_binding_rejects_cpu_tensors(lib):
    a = torch.zeros(8, 2, 64, dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        binding.rotary_fp16(a, a, torch.zeros(8, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(TypeError):
        binding.attention_fp16(a, a, a, i, 8)
    with pytest.raises(TypeError):
        binding.kv_read_u4(binding.kv_cache_u4(2, 1, 16, 64, device="cpu"), i, i, i, 1)
    with pytest.raises(ValueError):
        binding.rotary_fp16(a, a, i, torch.zeros(32), pairs="other")
