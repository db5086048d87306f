"""max_q lays the work out: the choice of pages is the same with any, attention is with any within the tolerances of test_gpu_serve.check_attention, and the same bits
come of the same call.  And the choice for the smallest queries."""
import numpy as np
import pytest
import torch

from tests import sparse_util as P
from tests.test_gpu_serve import attention_case, check_attention, dev, i32
from tests.test_gpu_sparse import choice_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


@pytest.mark.parametrize("n,kv", [([1] * 9, [5000, 1, 1300, 900, 128, 129, 2000, 640, 4000]), ([5, 1, 7, 40], [900, 2000, 7, 1500])])
@pytest.mark.parametrize("G,d", [(1, 64), (3, 128), (4, 128), (17, 64)])
def test_any_max_q(aq, n, kv, G, d):
    q, cu, cache, num, table = attention_case(n, kv, 2 * G, 2, d, G, tail=0)
    cache_d, table_d, qd = dev(cache.reshape(-1)), dev(table), q.cuda()
    slots = np.concatenate([table[b, :k // 128].astype(np.int64) * 128 + 127 for b, k in enumerate(kv)])
    summary = torch.zeros(num * aq.kv_summary_page_bytes(2, d), dtype=torch.uint8, device="cuda")
    aq.attnqat_kv_summarize(cache_d, dev(slots), summary, 2, d, num_pages=num)
    codes, scale = P.summary_parts(summary.cpu().numpy(), 2, d)
    want = P.select(q.double().numpy(), cu, codes, scale, table, kv, 2, 5, 1, 1)
    ref = P.attend(q.double().numpy(), cu, cache, table, kv, 2, want, d ** -0.5)
    for max_q in (None, 1, 2, 3, 5, max(n), 16, 1 << 40):
        blocks = aq.attnqat_kv_select(qd, i32(cu), summary, num, table_d, i32(kv), 2, 5, max_q=max_q)
        assert np.array_equal(blocks.cpu().numpy(), want), max_q
        two = [aq.attnqat_fwd_kv4_sparse(qd, i32(cu), cache_d, num, table_d, i32(kv), 2, blocks, max_q=max_q) for _ in range(2)]
        check_attention(*two[0], ref, max_q)
        assert torch.equal(two[0][0], two[1][0]) and torch.equal(two[0][1], two[1][1]), max_q


def test_choice_for_the_smallest_queries(aq):
    """Whole numbers below 16 times 2^-127, which the least power of two of the choice makes whole: q8 in proportion, so the choice is that of larger ones."""
    q, cu, table, num, codes, scale, summary = choice_case([1, 5], [3000, 2000], 4, 2, 64, 1, tail=0)
    k = np.random.default_rng(0).integers(-15, 16, tuple(q.shape)).astype(np.float64)
    q = torch.tensor(k * 2.0 ** -127).to(torch.bfloat16)
    assert np.array_equal(q.double().numpy(), k * 2.0 ** -127)
    got = aq.attnqat_kv_select(q.cuda(), i32(cu), dev(summary.reshape(-1)), num, dev(table), i32([3000, 2000]), 2, 6)
    assert np.array_equal(got.cpu().numpy(), P.select(q.double().numpy(), cu, codes, scale, table, [3000, 2000], 2, 6, 1, 1))
