"""CPU-only checks of the linear-layer and key/value-cache entry points: exports, refusals, and the
arithmetic of the binding's argument checks."""
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
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "b200kv.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(kv_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(binding.KV_EXPORTS)
    for name in names:
        assert getattr(lib, name) is not None


def epilogue(**kw):
    return ctypes.byref(binding._Epilogue(**kw))


def test_linear_refusals(lib):
    ok = dict(activation=0, c_is_fp16=1)
    assert lib.gemm_fp16_linear(0, 8, 8, 16, 16, 16, epilogue(**ok), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, None, epilogue(**ok), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, None, None) == -1
    assert lib.gemm_fp16_linear(8, 8, 12, 16, 16, 16, epilogue(**ok), None) == -2
    assert lib.gemm_fp16_linear(8, 8, 8, 24, 16, 16, epilogue(**ok), None) == -2
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 17, epilogue(**ok), None) == -2         # C off its element
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 18, epilogue(activation=0, c_is_fp16=0), None) == -2
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(activation=5, c_is_fp16=1), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(activation=0, c_is_fp16=2), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(ldc=7, **ok), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(residual=32, ldr=7, **ok), None) == -1
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(residual=16, ldr=9, **ok), None) == -1  # in place
    assert lib.gemm_fp16_linear(8, 8, 8, 16, 16, 16, epilogue(bias=18, **ok), None) == -2
    assert lib.gemm_s8_linear(8, 8, 16, 16, 16, None, 16, 16, epilogue(**ok), None) == -1
    assert lib.gemm_s8_linear(8, 8, 8, 16, 16, 16, 16, 16, epilogue(**ok), None) == -2
    assert lib.gemm_s8_linear(8, 8, 131072, 16, 16, 16, 16, 16, epilogue(**ok), None) == -3
    assert lib.gemm_s4_linear(8, 8, 16, 16, 16, 16, 16, 16, epilogue(**ok), None) == -2
    assert lib.gemm_s4_linear(8, 8, 32, 16, 16, 16, 18, 16, epilogue(**ok), None) == -2


def test_quantize_refusals(lib):
    assert lib.gemm_quantize_rows(0, 4, 32, 16, 0, 1, 16, 16, None) == -1
    assert lib.gemm_quantize_rows(1, 0, 32, 16, 0, 1, 16, 16, None) == -1
    assert lib.gemm_quantize_rows(1, 4, 32, None, 0, 1, 16, 16, None) == -1
    assert lib.gemm_quantize_rows(1, 4, 32, 16, 31, 1, 16, 16, None) == -1
    assert lib.gemm_quantize_rows(1, 4, 32, 16, 0, 2, 16, 16, None) == -1
    assert lib.gemm_quantize_rows(1, 4, 24, 16, 0, 1, 16, 16, None) == -2
    assert lib.gemm_quantize_rows(2, 4, 48, 16, 0, 1, 16, 16, None) == -2
    assert lib.gemm_quantize_rows(1, 4, 32, 17, 0, 1, 16, 16, None) == -2
    assert lib.gemm_quantize_rows(1, 4, 32, 18, 0, 0, 16, 16, None) == -2
    assert lib.gemm_quantize_rows(1, 4, 32, 16, 0, 1, 24, 16, None) == -2
    assert lib.gemm_quantize_rows(1, 4, 131072, 16, 0, 1, 16, 16, None) == -3


def cache(**kw):
    d = dict(k=16, v=16, k_scale=16, v_scale=16, num_pages=4, kv_heads=2, page_size=16, head_dim=64)
    d.update(kw)
    return ctypes.byref(binding._KvCache(**d))


def test_kv_refusals(lib):
    def append(c, batch=1, cu=16, past=16, table=16, stride=4, most=8, k=16, v=16, ts=128, hs=64):
        return lib.kv_append_s8(c, batch, cu, past, table, stride, most, k, v, ts, hs, None)

    def read(c, batch=1, cu=16, first=16, table=16, stride=4, most=8, k=16, v=16):
        return lib.kv_read_s8(c, batch, cu, first, table, stride, most, k, v, None)

    def attend(c, batch=1, cu=16, lens=16, table=16, stride=4, most=1, heads=4, q=16, ts=256, hs=64, scale=0.1,
               window=0, out=16, os=256):
        return lib.kv_attention_s8(c, batch, cu, lens, table, stride, most, heads, q, ts, hs, scale, window, out,
                                   os, None)

    for f in (append, read, attend):
        assert f(None) == -1
        for kw in (dict(k=None), dict(v_scale=None), dict(num_pages=0), dict(kv_heads=0), dict(page_size=8),
                   dict(page_size=48), dict(page_size=256), dict(head_dim=32), dict(head_dim=96)):
            assert f(cache(**kw)) == -1, kw
        assert f(cache(k=24)) == -2 and f(cache(k_scale=18)) == -2
        assert f(cache(), batch=0) == -1 and f(cache(), cu=None) == -1 and f(cache(), table=None) == -1
        assert f(cache(), stride=0) == -1 and f(cache(), most=0) == -1
        assert f(cache(), cu=18) == -2 and f(cache(), table=18) == -2
    assert append(cache(), k=None) == -1 and append(cache(), hs=32) == -1
    assert append(cache(), k=24) == -2 and append(cache(), ts=130) == -2
    assert read(cache(), k=None, v=None) == -1 and read(cache(), k=24) == -2
    assert attend(cache(), heads=3) == -1 and attend(cache(), heads=0) == -1 and attend(cache(), window=-1) == -1
    assert attend(cache(), scale=0.0) == -1 and attend(cache(), scale=float("nan")) == -1
    assert attend(cache(), out=None) == -1 and attend(cache(), os=128) == -1
    assert attend(cache(), q=24) == -2 and attend(cache(), hs=68) == -2


def test_binding_rejects_cpu_tensors(lib):
    a = torch.zeros(8, 16, dtype=torch.float16)
    with pytest.raises(TypeError):
        binding.gemm_fp16_linear(a, a, C=torch.zeros(8, 8, dtype=torch.float16))
    with pytest.raises(TypeError):
        binding.gemm_quantize_rows(a)
    with pytest.raises(TypeError):
        binding.kv_read_s8(binding.kv_cache_s8(2, 1, 16, 64, device="cpu"), a, a, a, 1)
