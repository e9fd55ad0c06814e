"""CPU-only: the cache entry points with a row count refuse what the forms without it refuse, and a count of none."""
import pytest

from paper_2608_10103_b200 import binding, build as lib_build
from test_kv_abi import cache


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


def test_refusals(lib):
    def append(c, rows=8, batch=1, ts=128):
        return lib.kv_append_s8_rows(c, batch, 16, 16, 16, 4, 8, 16, 16, ts, 64, rows, None)

    def read(c, rows=8, batch=1, k=16):
        return lib.kv_read_s8_rows(c, batch, 16, 16, 16, 4, 8, k, 16, rows, None)

    def attend(c, rows=8, batch=1, heads=4):
        return lib.kv_attention_s8_rows(c, batch, 16, 16, 16, 4, 1, heads, 16, 256, 64, 0.1, 0, 16, 256, rows, None)

    for f in (append, read, attend):
        assert f(None) == -1 and f(cache(page_size=8)) == -1 and f(cache(), batch=0) == -1
        assert f(cache(), rows=0) == -1 and f(cache(), rows=-1) == -1
        assert f(cache(k=24)) == -2
    assert append(cache(), ts=130) == -2 and read(cache(), k=24) == -2 and attend(cache(), heads=3) == -1
