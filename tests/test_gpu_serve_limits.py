"""Serving steps at the ends of their ranges."""
import pytest

from tests.test_gpu_serve import run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


@pytest.mark.parametrize("window", [1, 100, 130, 384, (1 << 20) - 1, 1 << 20, (1 << 31) - 200, (1 << 31) - 1])
@pytest.mark.parametrize("d", [64, 128])
def test_windows_with_more_queries_than_keys(aq, d, window):
    """Few rows and many; what lies before a sequence's first position is behind no window, however large."""
    run_attention(aq, [10, 3, 1, 40, 200, 7], [4, 0, 1, 0, 150, 300], 4, 2, d, window=window, seed=8)
