"""attnqat_kv_summarize where blocks of 16 keys' values have a NaN scale: they count as zeros, and no other value of the page is left out."""
import numpy as np
import pytest
import torch

from tests import serve_util as S, sparse_util as P
from tests.test_gpu_serve import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["one", "some", "a key", "all"])
@pytest.mark.parametrize("byte", [0x7F, 0xFF])
def test_nan_scales(d, how, byte):
    import paper_2603_00040_amd as aq
    rng = np.random.default_rng(d)
    num, Hkv = 3, 5
    cache = S.random_cache(num, Hkv, d, rng)
    nan = np.zeros((num, Hkv, 128, d // 16), bool)
    if how == "one":
        nan[0, 2, 77, d // 16 - 1] = nan[1, 0, 0, 0] = nan[2, 4, 127, 1] = True
    elif how == "a key":
        nan[:, :, 13] = True
    else:
        nan[:] = rng.random(nan.shape) < (0.1 if how == "some" else 2.0)
    scales, bad, zero = cache[:, :, 0, 64 * d:].reshape(nan.shape), cache.copy(), cache.copy()
    bad[:, :, 0, 64 * d:] = np.where(nan, byte, scales).reshape(num, Hkv, -1)
    zero[:, :, 0, 64 * d:] = np.where(nan, 0, scales).reshape(num, Hkv, -1)
    summary = torch.zeros(num * aq.kv_summary_page_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    aq.attnqat_kv_summarize(dev(bad.reshape(-1)), dev(np.arange(num, dtype=np.int64) * 128 + 127), summary, Hkv, d, num_pages=num)
    codes, scale = P.summary_parts(summary.cpu().numpy(), Hkv, d)
    for p in range(num):
        c, s = P.mean_of_page(zero, p, Hkv, d)
        assert np.array_equal(codes[p], c) and np.array_equal(scale[p], s), p
