"""The INT8 cache: windows wider than any sequence, and queries in front of the first token."""
import pytest

from paper_2608_10103_b200 import binding
from test_gpu_kv_attention import check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_state():
    yield
    assert binding.gemm_last_device_status() == 0


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4, 1000])
@pytest.mark.parametrize("news", [[8, 5, 2], [100, 70, 9]])
def test_wide_windows_over_short_sequences(news, window):
    """The first queries stand at positions below 0, from which a window may reach further down than 32 bits do."""
    check([4, 60, 1], news, 4, 2, 64, 16, window=window, seed=8)
