"""Serving steps at the ends of their ranges."""
import numpy as np
import pytest

from tests import serve_util as S
from tests.test_gpu_serve import check_attention, dev, i32, run_attention

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


def _cache_with_a_first_key(kv, gap, noise, Hkv, d, rng):
    """One sequence: the first key's score lies `gap` above the others' for a query of ones times gap / sqrt(d), and its value is zero; the others' values
    are 1 and 1.5, their keys zero or (noise) random."""
    num_pages = S.pages(kv)
    cache = np.zeros((num_pages, Hkv, 2, 128 * (d // 2 + d // 16)), np.uint8)
    cache[..., 64 * d:] = 56                                     # every scale 1
    codes, _ = S.parts(cache, Hkv, d)
    if noise:
        codes[:, :, 0] = rng.choice(np.array([0x00, 0x01, 0x10, 0x09, 0x90, 0x19, 0x91], np.uint8), codes[:, :, 0].shape)      # 0, +-0.5
    codes[:, :, 1] = rng.choice(np.array([0x22, 0x23, 0x32, 0x33], np.uint8), codes[:, :, 1].shape)
    codes[0, :, 0, 0] = 0x22
    codes[0, :, 1, 0] = 0
    return cache


@pytest.mark.parametrize("gap", [0.5, 12.0, 14.5, 15.7, 16.4, 17.0])
@pytest.mark.parametrize("noise", [False, True])
@pytest.mark.parametrize("B,n,kv,Hq,Hkv,d", [(100, 1, 2500, 16, 4, 128), (64, 4, 2500, 16, 4, 64), (1, 500, 4000, 16, 4, 128), (2, 300, 4000, 16, 4, 64)])
def test_a_first_key_that_draws_the_attention(aq, B, n, kv, Hq, Hkv, d, noise, gap):
    """What is left for the others decides o, which the first key adds nothing to.  A probability is rounded by a relative 2^-12 down to 2^-25 of a row's
    largest and by 2^-36 of the largest below.  The others' are 2^-24.6 (e^-17) of it on average or more, so that both together are at most
    (2^-12 + 2^-11.4) sum p |v| < 2^-10.5 sum p |v|: the bounds of check_attention."""
    rng = np.random.default_rng(7)
    cache = _cache_with_a_first_key(kv, gap, noise, Hkv, d, rng)
    table = np.tile(np.arange(cache.shape[0], dtype=np.int32), (B, 1))
    q = S.bf16(np.full((B * n, Hq, d), gap / np.sqrt(d)) * (1.0 - 0.02 * rng.random((B * n, Hq, 1))))
    cu = n * np.arange(B + 1)
    o, lse = aq.attnqat_fwd_kv4_ragged(q.cuda(), i32(cu), dev(cache.reshape(-1)), cache.shape[0], dev(table), i32([kv] * B), Hkv, True, max_q=n)
    check_attention(o, lse, S.attend(q.double().numpy(), cu, cache, table, [kv] * B, Hkv, True, 0, d ** -0.5), (B, n, d, noise, gap))
