"""attnqat_fwd_kv4_sparse where a tile's tokens and choices do not fill whole waves: tiles of 3, 5, 6, 7, 9 .. 15 tokens, whose last wave of choices has fewer lanes than the tile
has tokens, against 64 bits at the tolerances of attention over all pages.  Choices are pages of the row's own sequence, ascending, its own page last, as attnqat_kv_select gives
them."""
import numpy as np
import pytest
import torch

from tests import serve_util as S, sparse_util as P
from tests.test_gpu_serve import attention_case, check_attention, dev, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


def own_choice(n, kv, Hkv, n_blocks, rng):
    """For every row n_blocks pages of its sequence (all where there are no more), page 0 and its own page among them."""
    out = []
    for a, k in zip(n, kv):
        for i in range(a):
            last = (k - a + i) // 128
            for _ in range(Hkv):
                some = rng.permutation(np.arange(1, last))[:max(n_blocks - 2, 0)] if last > 1 else np.zeros(0, int)
                row = np.unique(np.concatenate([[0] if n_blocks > 1 else [], some, [last]]).astype(np.int32))
                out.append(np.concatenate([row, np.full(n_blocks - row.size, -1)]))
    return np.array(out, np.int32).reshape(-1, Hkv, n_blocks)


def run(aq, n, kv, Hq, Hkv, d, n_blocks, max_q, seed=0, tail=0):
    q, cu, cache, num, table = attention_case(n, kv, Hq, Hkv, d, seed, tail)
    blocks = own_choice(n, kv, Hkv, n_blocks, np.random.default_rng(seed + 1))
    # (rows behind the last sequence: zeros, as a program's buffer may have them)
    blocks = np.concatenate([blocks, np.zeros((tail, Hkv, n_blocks), np.int32)])
    T = q.shape[0]
    o, lse = torch.full((T, Hq, d), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, Hq), 5.0, device="cuda")
    aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), Hkv, dev(blocks), max_q=max_q, out=(o, lse))
    check_attention(o, lse, P.attend(q.double().numpy(), cu, cache, table, kv, Hkv, blocks, d ** -0.5), (n, kv, Hq, Hkv, d, n_blocks, max_q))
    if tail:
        assert bool((o[-tail:] == 5.0).all()) and bool((lse[-tail:] == 5.0).all())


# (heads of a group, max_q, pages of a row): tokens of a tile min(16 / G, max_q)
TILES = [(3, 8, 13), (3, 8, 26), (3, 8, 39), (3, 8, 52), (5, 8, 22), (5, 8, 43), (1, 3, 22), (4, 3, 43), (1, 5, 13), (2, 5, 26), (1, 6, 11), (2, 6, 54), (1, 7, 10), (2, 7, 19), (1, 9, 8),
         (1, 10, 20), (1, 11, 24), (1, 12, 6), (1, 13, 15), (1, 14, 28), (1, 15, 18), (1, 15, 60)]


@pytest.mark.parametrize("G,max_q,n_blocks", TILES)
@pytest.mark.parametrize("d", [64, 128])
def test_pieces(aq, G, max_q, n_blocks, d):
    """Tiles inside a sequence and across sequences."""
    n = [max_q, 1, max_q, 2, 2 * max_q + 1, 1, 1, max_q - 1]
    kv = [128 * n_blocks + 700, 128 * n_blocks - 5, max_q, 128 * n_blocks + 1, 300 + 64 * n_blocks, 1, 128 * n_blocks, 128 * n_blocks + 130]
    run(aq, n, kv, 2 * G, 2, d, n_blocks, max_q, seed=G + max_q + n_blocks)


@pytest.mark.parametrize("B,G,n_blocks", [(5, 3, 13), (13, 3, 26), (3, 5, 22), (7, 2, 10), (9, 1, 8), (15, 1, 13), (11, 1, 35)])
def test_single_tokens_without_max_q(aq, B, G, n_blocks):
    run(aq, [1] * B, [128 * n_blocks + 131 * b + 1 for b in range(B)], 2 * G, 2, 128, n_blocks, None, seed=B)


@pytest.mark.parametrize("T,n_blocks", [(150, 13), (300, 26)])
def test_units_that_fill_the_chip(aq, T, n_blocks):
    """Five drafted tokens a sequence, units of 16 and of 8 waves."""
    B = T // 5
    run(aq, [5] * B, [128 * n_blocks + 17 * b + 5 for b in range(B)], 24, 8, 64, n_blocks, 5, seed=T)


@pytest.mark.parametrize("n_blocks", [5, 9, 18, 22, 40])
@pytest.mark.parametrize("d,kv", [(64, [700000, 300, 690000, 1048576, 654321]), (128, [900000, 1048576, 800000, 1000, 1048500])])
def test_sequences_that_take_turns(aq, d, kv, n_blocks):
    """Sequences with more pages than a tile has room for together; a cache of few pages that the tables name many times."""
    rng = np.random.default_rng(d)
    num, n, T = 9, 3, 3 * len(kv)
    cache = S.random_cache(num, 1, d, rng)
    table = rng.integers(0, num, (len(kv), 8192)).astype(np.int32)
    q, cu = torch.randn(T, 1, d, generator=torch.Generator().manual_seed(d)).bfloat16(), np.arange(len(kv) + 1) * n
    # the reference: the pages chosen, as a sequence that has no others
    blocks, small = np.full((T, 1, n_blocks), -1, np.int32), np.full((T, 1, n_blocks), -1, np.int32)
    short, lens = np.zeros((len(kv), 60), np.int32), []
    for b, x in enumerate(kv):
        last = (x - 1) // 128
        some = np.unique(np.concatenate([rng.integers(0, last + 1, 58), [0, last]]))
        short[b, :some.size] = table[b, some]
        lens.append(x - 128 * (last + 1 - some.size))
        for i in range(n * b, n * b + n):
            at = np.sort(rng.permutation(some.size)[:n_blocks])
            at[-1] = some.size - 1
            small[i, 0, :at.size], blocks[i, 0, :at.size] = at, some[at]
    o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), 1, dev(blocks), max_q=16)
    check_attention(o, lse, P.attend(q.double().numpy(), cu, cache, short, lens, 1, small, d ** -0.5), (d, kv, n_blocks))


@pytest.mark.parametrize("G,max_q,n_blocks,tail", [(3, 8, 13, 4), (3, 8, 26, 9), (5, 8, 43, 2), (1, 7, 10, 6), (1, 15, 60, 13)])
def test_rows_behind_the_last_sequence(aq, G, max_q, n_blocks, tail):
    """They have no sequence, whatever their choice says, and keep what they hold."""
    run(aq, [1, max_q, 2], [128 * n_blocks, 128 * n_blocks + 77, 90], 2 * G, 2, 128, n_blocks, max_q, seed=tail, tail=tail)
    run(aq, [1], [128 * n_blocks + 3], 2 * G, 2, 64, n_blocks, None, seed=tail, tail=tail)
