"""attnqat_kv_summarize, attnqat_kv_select and attnqat_fwd_kv4_sparse: the first two against whole numbers (equal), attention against 64 bits at the tolerances
of attention over all pages (test_gpu_serve.check_attention: outputs rounded to bf16, probabilities to fp16)."""
import numpy as np
import pytest
import torch

from tests import serve_util as S, sparse_util as P
from tests.test_gpu_serve import _views, attention_case, check_attention, dev, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


# ------------------------------------------------------------------------------------------------------------ means
def check_means(aq, cache, num, Hkv, d, slots):
    """Pages that end in slots have their means, the rest of the summary is as it was."""
    size = num * aq.kv_summary_page_bytes(Hkv, d)
    summary = torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda")
    aq.attnqat_kv_summarize(dev(cache.reshape(-1)), dev(slots), summary, Hkv, d, num_pages=num)
    got = summary.cpu().numpy()
    codes, scale = P.summary_parts(got, Hkv, d)
    done = {int(s) // 128 for s in slots if 0 <= s < num * 128 and s % 128 == 127}
    for p in range(num):
        if p in done:
            c, s = P.mean_of_page(cache, p, Hkv, d)
            assert np.array_equal(codes[p], c) and np.array_equal(scale[p], s), p
        else:
            assert (codes[p] == 0x5A).all()
    assert (got.reshape(num, Hkv, d + 16)[..., d + 4:] == 0x5A).all()
    return codes, scale


@pytest.mark.parametrize("Hkv,d", [(1, 64), (3, 128), (8, 64)])
@pytest.mark.parametrize("T", [1, 15, 16, 17, 64, 65, 300])
def test_means(aq, Hkv, d, T):
    rng = np.random.default_rng(T + d)
    num = 9
    cache = S.random_cache(num, Hkv, d, rng)
    slots = rng.integers(0, num, T).astype(np.int64) * 128 + np.where(rng.random(T) < 0.5, 127, rng.integers(0, 127, T))
    slots[rng.random(T) < 0.1] = rng.choice([-1, num * 128 + 127, 1 << 40, -129])
    check_means(aq, cache, num, Hkv, d, slots)


@pytest.mark.parametrize("kind", ["zeros", "largest", "least", "one", "ties", "cancel"])
@pytest.mark.parametrize("d", [64, 128])
def test_means_at_the_ends_of_the_range(aq, kind, d):
    cache = np.zeros((2, 2, 2, 128 * (d // 2 + d // 16)), np.uint8)
    codes, scales = cache[..., :64 * d], cache[..., 64 * d:]
    k = codes[:, :, 0].reshape(2, 2, 128, d // 2)
    if kind == "largest":                                          # 6 * 448, every second channel negative: sums of 128 * 2688 2^10 < 2^29
        k[:], scales[:] = 0xF7, 0x7E
    elif kind == "least":
        k[:, :, 5, 3], scales[:] = 0x01, 0x01                      # one value of 2^-10
    elif kind == "one":
        k[:], scales[:] = 0x22, 0x38                               # all 1
    elif kind == "ties":                                           # sums 127.5, 126.5, ... of the largest code's unit
        scales[:] = 0x38
        k[:, :, :, :] = 0x02                                       # even channels 1: 128
        k[:, :, 0, 1], k[:, :, 0, 2], k[:, :, :2, 3] = 0x01, 0x0A, 0x01                         # 127.5, 126, 127
    elif kind == "cancel":
        scales[:] = 0x7E
        k[:, :, 0::2], k[:, :, 1::2] = 0x77, 0xFF
        k[:, :, 0, 7] = 0x76                                       # one channel is left over
    check_means(aq, cache, 2, 2, d, np.array([127, 255], np.int64))


def test_means_of_a_long_prompt(aq):
    """Enough rows for the wider launch."""
    rng = np.random.default_rng(3)
    num, Hkv, d = 80, 2, 64
    cache = S.random_cache(num, Hkv, d, rng)
    pages = rng.permutation(num)[:70]
    slots = (pages[:, None].astype(np.int64) * 128 + np.arange(128)).reshape(-1)[37:]
    check_means(aq, cache, num, Hkv, d, slots[:-5])


# ------------------------------------------------------------------------------------------------------------ choice
def choice_case(n, kv, Hq, Hkv, d, seed, tail=2, few=False):
    """Queries, and means of every page: codes of few different values (few: scores that are equal)."""
    rng = np.random.default_rng(seed)
    table, num = S.make_table([max(k, 1) for k in kv], rng)
    cu = np.concatenate([[0], np.cumsum(n)])
    q = S.bf16(rng.standard_normal((int(cu[-1]) + tail, Hq, d)) * np.exp2(rng.integers(-9, 9, (int(cu[-1]) + tail, 1, 1))))
    codes = rng.integers(-1, 2, (num, Hkv, d)).astype(np.int8) if few else rng.integers(-127, 128, (num, Hkv, d)).astype(np.int8)
    if few:
        codes[:] = codes[rng.integers(0, 3, num)]
    scale = np.exp2(rng.integers(-10, -7, (num, Hkv))).astype(np.float32) if not few else np.full((num, Hkv), 2.0 ** -9, np.float32)
    summary = rng.integers(0, 256, (num, Hkv, d + 16)).astype(np.uint8)
    summary[..., :d] = codes.view(np.uint8)
    summary[..., d:d + 4] = np.ascontiguousarray(scale)[..., None].view(np.uint8)
    return q, cu, table, num, codes, scale, summary


def run_choice(aq, n, kv, Hq, Hkv, d, n_blocks, first=1, last=1, seed=0, few=False, layout="plain", max_q=None, holes=False):
    q, cu, table, num, codes, scale, summary = choice_case(n, kv, Hq, Hkv, d, seed, few=few)
    if holes:
        table[:, ::3] = np.where(np.arange(table.shape[0])[:, None] % 2, -1, num + 5)
    out = torch.full((q.shape[0], Hkv, n_blocks), -7, dtype=torch.int32, device="cuda")
    got = aq.attnqat_kv_select(_views(q.cuda(), layout), i32(cu), dev(summary.reshape(-1)), num, dev(table), i32(kv), Hkv, n_blocks, first=first, last=last,
                               max_q=max_q or max(max(n), 1), out=out)
    want = P.select(q.double().numpy(), cu, codes, scale, table, kv, Hkv, n_blocks, first, last)
    assert np.array_equal(got.cpu().numpy(), want), (n, kv, Hq, Hkv, d, n_blocks, first, last)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 9, 16, 17, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_choice_for_heads_of_a_group(aq, G, d):
    run_choice(aq, [1, 3, 1], [2600, 1900, 4000], 2 * G, 2, d, 6, seed=G)
    run_choice(aq, [1, 3, 1], [2600, 1900, 4000], G, 1, d, 5, seed=G, few=True)


@pytest.mark.parametrize("kv", [[1], [127], [128], [129], [256], [257], [640], [641], [768], [769], [8192], [8321], [20000], [1, 700, 128, 3000]])
@pytest.mark.parametrize("n_blocks,first,last", [(1, 0, 1), (5, 1, 1), (5, 0, 5), (5, 4, 1), (64, 1, 2)])
def test_choice_for_one_query(aq, kv, n_blocks, first, last):
    run_choice(aq, [1] * len(kv), kv, 4, 2, 128, n_blocks, first, last, seed=kv[0])
    run_choice(aq, [1] * len(kv), kv, 4, 2, 64, n_blocks, first, last, seed=kv[0], few=True, holes=True)


@pytest.mark.parametrize("n,kv", [([1, 7, 3, 16, 2], [1000, 7, 1500, 16, 3131]), ([129, 1, 64], [129, 4000, 1700]), ([0, 4, 0, 0, 9, 0], [50, 600, 0, 1280, 900, 3]),
                                  ([10, 3, 40], [4, 0, 2500]), ([300], [2111]), ([1] * 70, [900] * 70)])
@pytest.mark.parametrize("Hq,Hkv,d,layout", [(8, 2, 128, "plain"), (3, 3, 64, "fused"), (16, 1, 128, "heads")])
@pytest.mark.parametrize("few", [False, True])
def test_choice_ragged(aq, n, kv, Hq, Hkv, d, layout, few):
    run_choice(aq, n, kv, Hq, Hkv, d, 4, seed=sum(n), layout=layout, few=few)
    run_choice(aq, n, kv, Hq, Hkv, d, 7, 2, 3, seed=sum(n), layout=layout, few=few, max_q=1)


def test_choice_of_many(aq):
    run_choice(aq, [2, 1], [40000, 70000], 4, 1, 64, 200, seed=1)
    run_choice(aq, [1], [150000], 4, 1, 64, 1024, 3, 5, seed=1)
    run_choice(aq, [1, 2], [300, 131073], 2, 1, 64, 1000, 0, 1, seed=2, few=True)


@pytest.mark.parametrize("q_scale", [0.0, 2.0 ** -100, 2.0 ** 100])
def test_choice_for_queries_far_from_one(aq, q_scale):
    q, cu, table, num, codes, scale, summary = choice_case([1, 5], [3000, 2000], 4, 2, 64, 1, tail=0)
    q = (q.double() * q_scale).to(torch.bfloat16)
    got = aq.attnqat_kv_select(q.cuda(), i32(cu), dev(summary.reshape(-1)), num, dev(table), i32([3000, 2000]), 2, 6)
    assert np.array_equal(got.cpu().numpy(), P.select(q.double().numpy(), cu, codes, scale, table, [3000, 2000], 2, 6, 1, 1))


def test_choice_stays_inside_whatever_comes(aq):
    """NaN and infinite queries, scales of nothing, offsets and lengths out of range: page numbers of the sequence, ascending, no row twice."""
    q, cu, table, num, codes, scale, summary = choice_case([3, 2, 4], [3000, 2000, 1280], 4, 2, 64, 1, tail=0)
    q[0, 1, 5], q[3, 0, 0], q[5] = float("nan"), float("inf"), float("-inf")
    summary[::2, :, 64:68] = 0xFF
    table = np.clip(table, 0, num - 1)
    for c, lens in (([0, 3, 5, 9], [3000, 2000, 1280]), ([-5, 4, 2, 400], [3000, 2000, 1280]), ([0, 3, 5, 9], [-7, 1 << 30, 1 << 20])):
        out = torch.full((9, 2, 6), -7, dtype=torch.int32, device="cuda")
        aq.attnqat_kv_select(q.cuda(), i32(c), dev(summary.reshape(-1)), num, dev(table), i32(lens), 2, 6, out=out)
        got = out.cpu().numpy()
        for row in got.reshape(-1, 6):
            if row[0] == -7:
                assert (row == -7).all()
                continue
            real = row[row >= 0]
            assert (np.diff(real) > 0).all() and (real < table.shape[1]).all() and (row[len(real):] == -1).all()


# ------------------------------------------------------------------------------------------------------------ attention
def random_blocks(T, Hkv, n_blocks, most, rng):
    """Any choice: in no order, with pages twice, behind the row and none at all."""
    blocks = rng.integers(0, most + 2, (T, Hkv, n_blocks)).astype(np.int32)
    blocks[rng.random(blocks.shape) < 0.2] = -1
    blocks[rng.random(blocks.shape) < 0.02] = 1 << 30
    blocks[rng.random(blocks.shape) < 0.02] = -(1 << 31)
    if T > 3:
        blocks[2] = -1
    return blocks


def run_sparse(aq, n, kv, Hq, Hkv, d, n_blocks, seed=0, tail=3, layout="plain", max_q=None, scale=None, q_scale=1.0, blocks=None, spread=False):
    q, cu, cache, num, table = attention_case(n, kv, Hq, Hkv, d, seed, tail, q_scale)
    T = q.shape[0]
    rng = np.random.default_rng(seed + 1)
    if blocks is None:
        blocks = random_blocks(T, Hkv, n_blocks, max(S.pages(k) for k in kv), rng)
    o, lse = _views(torch.full((T, Hq, d), 5.0, dtype=torch.bfloat16, device="cuda"), layout), torch.full((T, Hq), 5.0, device="cuda")
    aq.attnqat_fwd_kv4_sparse(_views(q.cuda(), layout), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), Hkv, dev(blocks), max_q=max_q or max(max(n), 1), scale=scale, out=(o, lse))
    check_attention(o, lse, P.attend(q.double().numpy(), cu, cache, table, kv, Hkv, blocks, d ** -0.5 if scale is None else scale, spread), (n, kv, Hq, Hkv, d))
    if tail:
        assert bool((o[-tail:] == 5.0).all()) and bool((lse[-tail:] == 5.0).all())
    return o, lse


@pytest.mark.parametrize("kv", [[1], [2], [31], [33], [127], [128], [129], [255], [257], [1000], [4097], [1, 128, 5, 640, 33]])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("n_blocks", [1, 4, 40])
def test_one_query(aq, kv, Hq, Hkv, d, n_blocks):
    run_sparse(aq, [1] * len(kv), kv, Hq, Hkv, d, n_blocks, seed=len(kv) + kv[0])


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 15, 16, 17, 32, 33, 71])
def test_heads_of_a_group(aq, G):
    run_sparse(aq, [1, 1, 6], [300, 77, 700], 2 * G, 2, 64 if G % 2 else 128, 3, seed=G)


@pytest.mark.parametrize("n,kv", [([1, 7, 3, 16, 2], [1, 7, 500, 16, 131]), ([5, 100, 1], [5, 100, 1]), ([129, 1, 64], [129, 400, 700]), ([300], [1111]),
                                  ([0, 4, 0, 0, 9, 0], [50, 60, 0, 128, 9, 3]), ([1] * 40, [300] * 40), ([10, 3, 40, 20], [4, 0, 0, 150])])
@pytest.mark.parametrize("Hq,Hkv,d,layout", [(8, 2, 128, "plain"), (6, 2, 64, "fused"), (1, 1, 128, "heads"), (4, 4, 64, "plain")])
@pytest.mark.parametrize("max_q", [None, 1, 2])
def test_ragged(aq, n, kv, Hq, Hkv, d, layout, max_q):
    run_sparse(aq, n, kv, Hq, Hkv, d, 5, seed=sum(n), layout=layout, max_q=max_q)


@pytest.mark.parametrize("Hq,Hkv,d,T", [(32, 8, 128, 1050), (8, 8, 64, 1030), (16, 8, 128, 1040), (24, 8, 64, 1100), (40, 8, 128, 900), (64, 8, 64, 520), (72, 8, 128, 400), (128, 8, 128, 270),
                                        (160, 8, 64, 150), (264, 8, 128, 130)])
@pytest.mark.parametrize("kind", ["random", "alike", "all"])
def test_many_rows(aq, Hq, Hkv, d, T, kind):
    """Long pieces beside single tokens, sequences without rows and rows without a key, in one step; any choice of pages, nearly the same one for all rows, and every page."""
    n, kv = [1, 0, T // 2, 3, 17, 0, T - T // 2 - 61, 40], [700, 50, T // 2 + 300, 2, 1900, 0, T - T // 2 - 61, 23]
    q, cu, cache, num, table = attention_case(n, kv, Hq, Hkv, d, T, 0)
    rng = np.random.default_rng(T)
    most = max(S.pages(k) for k in kv)
    blocks = random_blocks(T, Hkv, 5, most, rng)
    if kind == "alike":
        blocks[:] = np.where(rng.random(blocks.shape) < 0.9, np.array([0, 2, 1, 2, 3], np.int32), blocks)
    elif kind == "all":
        blocks = np.broadcast_to(np.arange(most, dtype=np.int32), (T, Hkv, most)).copy()
    o, lse = run_sparse(aq, n, kv, Hq, Hkv, d, blocks.shape[2], seed=T, tail=0, blocks=blocks)
    few = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), Hkv, dev(blocks), max_q=1)      # (a token to a tile)
    ref = P.attend(q.double().numpy(), cu, cache, table, kv, Hkv, blocks, d ** -0.5)
    check_attention(*few, ref, "few")
    again = run_sparse(aq, n, kv, Hq, Hkv, d, blocks.shape[2], seed=T, tail=0, blocks=blocks, layout="fused")
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("q_scale", [0.0, 1e-30, 40.0])
def test_many_rows_whose_scores_spread(aq, q_scale):
    """References that stay, and that follow at almost every page."""
    for d in (64, 128):
        run_sparse(aq, [1100, 20], [3000, 700], 32, 8, d, 9, seed=3, q_scale=q_scale, scale=0.02 if q_scale > 1 else None, spread=True)


def test_nan_stays_in_its_row_among_many(aq):
    n, kv, G = [1030, 60], [1100, 400], 4
    q, cu, cache, num, table = attention_case(n, kv, 8 * G, 8, 128, 1, tail=0)
    blocks = dev(random_blocks(sum(n), 8, 4, 9, np.random.default_rng(1)))
    args = (i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), 8, blocks)
    qd = q.cuda()
    o, lse = aq.attnqat_fwd_kv4_sparse(qd, *args, max_q=max(n))
    qn = qd.clone()
    at = int((lse[:, 9] > -1e30).nonzero()[500])
    qn[at, 9, 17] = float("nan")
    on, ln = aq.attnqat_fwd_kv4_sparse(qn, *args, max_q=max(n))
    assert bool(on[at, 9].isnan().all()) and bool(ln[at, 9].isnan())
    on[at, 9], ln[at, 9] = o[at, 9], lse[at, 9]
    assert torch.equal(on, o) and torch.equal(ln, lse)


@pytest.mark.parametrize("n,T", [(1, 1), (900, 900), (3000, 3000)])
def test_few_and_many_rows(aq, n, T):
    """Split pages and whole ones."""
    run_sparse(aq, [n], [max(n, 1500)], 4, 1, 64, 3, seed=n, tail=1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,n", [(32, 1), (29, 1), (32, 4), (64, 1), (58, 2), (57, 4)])
@pytest.mark.parametrize("n_blocks", [2, 90])
def test_steps_that_fill_the_chip(aq, d, B, n, n_blocks):
    """Single and drafted tokens, as many as workgroups of 16 or 8 waves for a unit have room: long lists of pages beside sequences of nothing, one key and less than their rows."""
    kv = [0, 1, 12000, 127, 128, 129, 11777] + [n + 61 * b for b in range(B - 7)]
    kv[9] = max(n - 1, 1)
    run_sparse(aq, [n] * B, kv, 32, 8, d, n_blocks, seed=B + n, tail=0 if n > 1 else 3)


def test_many_pages(aq):
    run_sparse(aq, [1, 5], [9000, 17001], 4, 1, 64, 300, seed=4)
    run_sparse(aq, [2], [140000], 2, 1, 64, 1024, seed=5)
    run_sparse(aq, [20], [140000], 1, 1, 128, 70, seed=6)


@pytest.mark.parametrize("d,kv", [(64, [700000, 300, 690000, 1048576, 654321]), (128, [900000, 1048576, 800000, 1000, 1048500])])
def test_long_sequences_that_share_a_tile(aq, d, kv):
    """More pages than the tokens of a tile find room for together: few of them chosen, and a cache of few pages that the tables name many times."""
    rng = np.random.default_rng(d)
    num, n_blocks, n, T = 9, 40, 3, 3 * len(kv)
    cache = S.random_cache(num, 1, d, rng)
    table = rng.integers(0, num, (len(kv), 8192)).astype(np.int32)
    q, cu = torch.randn(T, 1, d, generator=torch.Generator().manual_seed(d)).bfloat16(), np.arange(len(kv) + 1) * n
    # the pages that may be chosen, and the same choice of a sequence that has no others
    blocks, small = np.full((T, 1, n_blocks), -1, np.int32), np.full((T, 1, n_blocks), -1, np.int32)
    short, lens = np.zeros((len(kv), 60), np.int32), []
    for b, x in enumerate(kv):
        last = (x - 1) // 128
        some = np.unique(np.append(rng.integers(0, last + 1, 59), last))
        short[b, :some.size] = table[b, some]
        lens.append(x - 128 * (last + 1 - some.size))
        for i in range(n * b, n * b + n):
            at = rng.integers(0, some.size, n_blocks)
            small[i, 0], blocks[i, 0] = at, some[at]
    o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), 1, dev(blocks), max_q=16)
    check_attention(o, lse, P.attend(q.double().numpy(), cu, cache, short, lens, 1, small, d ** -0.5), (d, kv))


@pytest.mark.parametrize("q_scale,scale", [(1e-38, None), (1e30, 1e-31), (0.0, None), (1.0, 0.4), (1.0, 1e-44)])
def test_scales(aq, q_scale, scale):
    run_sparse(aq, [1, 20], [200, 300], 4, 2, 128, 3, seed=3, q_scale=q_scale, scale=scale)


def test_all_pages_are_attention_over_the_cache(aq):
    """Every page chosen: what attnqat_fwd_kv4_ragged computes (both rounded to bf16, with probabilities in fp16)."""
    for n, kv, G, d in (([1, 1, 1], [3000, 40, 900], 4, 128), ([50, 1, 20], [700, 500, 60], 2, 64)):
        q, cu, cache, num, table = attention_case(n, kv, 2 * G, 2, d, 5, tail=0)
        most = table.shape[1]
        blocks = np.broadcast_to(np.arange(most, dtype=np.int32), (q.shape[0], 2, most))
        args = (q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), 2)
        o, lse = aq.attnqat_fwd_kv4_sparse(*args, dev(blocks), max_q=max(n))
        ref = S.attend(q.double().numpy(), cu, cache, table, kv, 2, True, 0, d ** -0.5)
        check_attention(o, lse, ref)
        check_attention(*aq.attnqat_fwd_kv4_ragged(*args, True, max_q=max(n)), ref)


def test_nan_stays_in_its_row(aq):
    for n, G in (([1, 3], 4), ([60, 40], 2), ([5, 4], 1)):
        q, cu, cache, num, table = attention_case(n, [300, 200], 2 * G, 2, 128, 1, tail=0)
        blocks = dev(np.broadcast_to(np.arange(3, dtype=np.int32), (sum(n), 2, 3)))
        args = (i32(cu), dev(cache.reshape(-1)), num, dev(table), i32([300, 200]), 2, blocks)
        qd = q.cuda()
        o, lse = aq.attnqat_fwd_kv4_sparse(qd, *args, max_q=max(n))
        qn = qd.clone()
        qn[1, 2 * G - 1, 17] = float("nan")
        on, ln = aq.attnqat_fwd_kv4_sparse(qn, *args, max_q=max(n))
        assert bool(on[1, 2 * G - 1].isnan().all()) and bool(ln[1, 2 * G - 1].isnan())
        on[1, 2 * G - 1], ln[1, 2 * G - 1] = o[1, 2 * G - 1], lse[1, 2 * G - 1]
        assert torch.equal(on, o) and torch.equal(ln, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("G,max_q", [(1, 16), (4, 4), (2, 1), (17, 4)])
def test_nan_in_the_cache_reaches_the_rows_that_see_it(aq, which, d, G, max_q):
    """A NaN scale of one key: rows of other sequences, rows that did not choose its page and rows before it keep their bits; of V only its 16 channels turn to NaN."""
    n, kv, Hkv = [1, 5, 1, 8, 1, 1], [500, 300, 380, 390, 700, 40], 2
    q, cu, cache, num, table = attention_case(n, kv, G * Hkv, Hkv, d, 7, tail=0)
    T = q.shape[0]
    rng = np.random.default_rng(3)
    blocks = np.stack([np.sort(rng.permutation(4)[:3]) for _ in range(T * Hkv)]).reshape(T, Hkv, 3).astype(np.int32)
    run = lambda c: aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(c.reshape(-1)), num, dev(table), i32(kv), Hkv, dev(blocks), max_q=max_q)  # noqa: E731
    o, lse = run(cache)
    assert not bool(o.isnan().any())
    for b, key, block in ((1, 260, 0), (3, 386, d // 16 - 1), (3, 100, 2), (4, 17, 1), (4, 255, d // 16 - 1), (0, 499, 1)):
        bad = cache.copy()
        half = 64 * d + 128 * (d // 16)                            # codes and scales of K, then of V
        row = bad.reshape(num, Hkv, 2 * half)[table[b, key // 128], 1]
        row[(which == "V") * half + 64 * d + key % 128 * (d // 16) + block] = 0x7F
        got, gl = run(bad)
        sees = torch.zeros(T, dtype=torch.bool)
        for i in range(n[b]):
            sees[cu[b] + i] = key <= kv[b] - n[b] + i and key // 128 in blocks[cu[b] + i, 1]
        hit = torch.zeros(o.shape, dtype=torch.bool)
        hit[sees, G:, 16 * block if which == "V" else 0:16 * block + 16 if which == "V" else d] = True
        assert torch.equal(got.isnan().cpu(), hit), (b, key)
        hit = hit.cuda()
        assert torch.equal(torch.where(hit, 0, got), torch.where(hit, 0, o)), (b, key)
        if which == "V":
            assert torch.equal(gl, lse)
        else:
            at = torch.zeros(lse.shape, dtype=torch.bool)
            at[sees, G:] = True
            assert torch.equal(gl.isnan().cpu(), at) and torch.equal(torch.where(at.cuda(), 0, gl), torch.where(at.cuda(), 0, lse))


def test_nan_queries_without_a_page(aq):
    """A row that chose nothing beside rows that did: 0 and -inf, whatever its query is."""
    n, kv = [6, 1, 1], [400, 300, 200]
    q, cu, cache, num, table = attention_case(n, kv, 8, 2, 128, 3, tail=0)
    q[2], q[6, :4], q[7, 5] = float("nan"), float("inf"), float("-inf")
    blocks = np.broadcast_to(np.array([0, 1], np.int32), (8, 2, 2)).copy()
    blocks[2], blocks[6, 0], blocks[7] = -1, 99, -5
    for max_q in (1, 4):
        o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32(kv), 2, dev(blocks), max_q=max_q)
        none = torch.zeros((8, 8), dtype=torch.bool, device="cuda")
        none[2], none[6, :4], none[7] = True, True, True
        assert bool((o[none] == 0).all()) and bool((lse[none] == float("-inf")).all())
        assert not bool(o[~none].isnan().any()) and bool(lse[~none].isfinite().all())


def test_pages_outside_the_cache_read_as_zeros(aq):
    q, cu, cache, num, table = attention_case([1, 20], [700, 300], 4, 2, 128, 2)
    table[0, 2], table[1, 0], table[0, 4] = -1, num, 1 << 30
    blocks = np.broadcast_to(np.array([4, 2, 0, 5, 1], np.int32), (q.shape[0], 2, 5))
    o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(cu), dev(cache.reshape(-1)), num, dev(table), i32([700, 300]), 2, dev(blocks))
    check_attention(o, lse, P.attend(q.double().numpy(), cu, cache, table, [700, 300], 2, blocks, 128 ** -0.5))


def test_without_lse_and_padding_rows(aq):
    q, cu, cache, num, table = attention_case([1, 20], [700, 300], 4, 2, 128, 2, tail=11)
    blocks = dev(np.broadcast_to(np.arange(3, dtype=np.int32), (q.shape[0], 2, 3)))
    args = (i32(cu), dev(cache.reshape(-1)), num, dev(table), i32([700, 300]), 2)
    o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), *args, blocks)
    o2 = torch.empty_like(o)
    aq.attnqat_fwd_kv4_sparse(q.cuda(), *args, blocks, out=(o2, None))
    assert torch.equal(o[:21], o2[:21])


@pytest.mark.parametrize("n,kv", [([1, 1, 4], [3000, 40, 900]), ([300, 1, 20], [700, 500, 60])])
def test_same_bits_again_on_another_stream_and_in_graphs(aq, n, kv):
    """Selection and attention; two graphs that share a workspace, replayed in turn."""
    Hq, Hkv, d = 8, 2, 128
    q, cu, cache, num, table = attention_case(n, kv, Hq, Hkv, d, 5, tail=0)
    cache_d, slots = dev(cache.reshape(-1)), dev(np.concatenate([table[b, :k // 128].astype(np.int64) * 128 + 127 for b, k in enumerate(kv)]))
    summary = torch.zeros(num * aq.kv_summary_page_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    qd, T = q.cuda(), q.shape[0]
    step = (i32(cu), dev(table), i32(kv))
    ws = torch.empty(aq.kv4_sparse_workspace_bytes(T, Hq, Hkv, max(n), 4, d), dtype=torch.uint8, device="cuda")

    def run(out):
        aq.attnqat_kv_summarize(cache_d, slots, summary, Hkv, d, num_pages=num)
        aq.attnqat_kv_select(qd, step[0], summary, num, step[1], step[2], Hkv, 4, max_q=max(n), out=out[0])
        aq.attnqat_fwd_kv4_sparse(qd, step[0], cache_d, num, step[1], step[2], Hkv, out[0], max_q=max(n), workspace=ws, out=out[1:])

    new = lambda: (torch.zeros((T, Hkv, 4), dtype=torch.int32, device="cuda"), torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hq), device="cuda"))  # noqa: E731
    want, out, other = new(), new(), new()
    run(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for gr, x in zip(graphs, (out, other)):
        with torch.cuda.graph(gr):
            run(x)
    for i in range(3):
        qd.mul_(-0.75)
        run(want)
        for x in (*out, *other):
            x.zero_()
        ws.random_(0, 256)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, out, other)), i


def test_offsets_beyond_32_bits(aq):
    Hkv, d = 8, 128
    page = aq.kv_cache_page_bytes_nvfp4(Hkv, d)
    num = (5 << 30) // page
    cache = torch.zeros(num * page, dtype=torch.uint8, device="cuda")
    summary = torch.zeros(num * aq.kv_summary_page_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(6)
    kv, n = [700], [3]
    table = np.array([[num - 1, 3, num - 7, num // 2, num - 2, num - 3]], np.int32)
    pos = np.arange(700)
    slots = table[0, pos // 128].astype(np.int64) * 128 + pos % 128
    x = S.bf16(rng.standard_normal((2, 700, Hkv, d)))
    aq.attnqat_kv_cache_append(x[0].cuda(), x[1].cuda(), cache, dev(slots))
    aq.attnqat_kv_summarize(cache, dev(slots), summary, Hkv, d)
    used = sorted(set(table.reshape(-1)))
    at = torch.tensor(used, device="cuda")
    small, small_s = cache.view(num, -1)[at].cpu().numpy().reshape(len(used), Hkv, 2, -1), summary.view(num, -1)[at].cpu().numpy()      # the reference: those pages alone
    table_s = np.array([[used.index(t) for t in row] for row in table], np.int32)
    codes, scale = P.summary_parts(small_s.reshape(-1), Hkv, d)
    for p in table_s[0, :5]:
        c, s = P.mean_of_page(small, p, Hkv, d)
        assert np.array_equal(codes[p], c) and np.array_equal(scale[p], s)
    q = S.bf16(rng.standard_normal((3, 16, d)))
    blocks = aq.attnqat_kv_select(q.cuda(), i32([0, 3]), summary, num, dev(table), i32(kv), Hkv, 4)
    want = P.select(q.double().numpy(), [0, 3], codes, scale, table_s, kv, Hkv, 4, 1, 1)
    assert np.array_equal(blocks.cpu().numpy(), want)
    o, lse = aq.attnqat_fwd_kv4_sparse(q.cuda(), i32([0, 3]), cache, num, dev(table), i32(kv), Hkv, blocks)
    check_attention(o, lse, P.attend(q.double().numpy(), [0, 3], small, table_s, kv, Hkv, want, d ** -0.5))


def test_offsets_out_of_order_stay_inside(aq):
    q, cu, cache, num, table = attention_case([3, 2, 4], [30, 20, 128], 4, 2, 64, 1, tail=0)
    blocks = dev(np.zeros((9, 2, 2), np.int32))
    for c, lens in (([-5, 4, 2, 400], [30, 20, 128]), ([0, 3, 5, 9], [-7, 1 << 30, 1 << 20])):
        o = torch.full((11, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        aq.attnqat_fwd_kv4_sparse(q.cuda(), i32(c), dev(cache.reshape(-1)), num, dev(np.clip(table, 0, num - 1)), i32(lens), 2, blocks, out=(o[1:10], None))
        torch.cuda.synchronize()
        assert bool((o[0] == 5.0).all()) and bool((o[10] == 5.0).all())


def test_many_sequences(aq):
    rng = np.random.default_rng(31)
    for B in (300, 700):
        kv = [int(x) for x in rng.integers(0, 700, B)]
        n = [min(k, int(rng.choice([0, 1, 1, 1, 2]))) for k in kv]
        run_choice(aq, n, kv, 2, 1, 64, 3, seed=B)
        run_sparse(aq, n, kv, 2, 1, 64, 3, seed=B)


def test_nothing_to_do_leaves_the_outputs(aq):
    q, cu, cache, num, table = attention_case([3, 2], [30, 20], 4, 2, 64, 1, tail=0)
    o, lse, blocks = torch.full((5, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 4), 5.0, device="cuda"), torch.full((5, 2, 3), 9, dtype=torch.int32, device="cuda")
    summary = torch.zeros(num * aq.kv_summary_page_bytes(2, 64), dtype=torch.uint8, device="cuda")
    cu, table, lens, cache = i32([0, 0, 0]), dev(table), i32([30, 20]), dev(cache.reshape(-1))
    aq.attnqat_kv_select(q.cuda(), cu, summary, num, table, lens, 2, 3, out=blocks)
    aq.attnqat_fwd_kv4_sparse(q.cuda(), cu, cache, num, table, lens, 2, blocks, out=(o, lse))
    assert bool((o == 5.0).all()) and bool((lse == 5.0).all()) and bool((blocks == 9).all())
    none = q[:0].cuda()
    assert aq.attnqat_kv_select(none, cu, summary, num, table, lens, 2, 3).shape == (0, 2, 3)
    assert aq.attnqat_fwd_kv4_sparse(none, cu, cache, num, table, lens, 2, blocks[:0])[0].shape == (0, 4, 64)
    aq.attnqat_kv_summarize(cache, torch.zeros(0, dtype=torch.int64, device="cuda"), summary, 2, 64)


# ------------------------------------------------------------------------------------------------------------ together
def test_steps_of_a_server(aq):
    """Plan, append with rotary positions, summarize, select, attend, step after step, as one captured graph from the fourth on; every step against a plain
    server that keeps what was appended."""
    rng = np.random.default_rng(23)
    B, Hq, Hkv, d, most, num, T, nb = 5, 8, 2, 128, 9, 30, 700, 4
    e = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    lens, want, table, ring, state = e(B), e(B), torch.full((B, most), -1, dtype=torch.int32, device="cuda"), i32(rng.permutation(num)), i32([5, num, 0])
    cu, slots, positions = e(B + 1), e(T, torch.int64), e(T)
    cache, summary = dev(rng.integers(0, 256, num * aq.kv_cache_page_bytes_nvfp4(Hkv, d), dtype=np.uint8)), e(num * aq.kv_summary_page_bytes(Hkv, d), torch.uint8)
    qkv = torch.zeros((T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=1)
    rope = aq.rope_table((d,), theta=500000.0, layout="halves")
    freqs, axis = [500000.0 ** (-2.0 * i / d) for i in range(d // 2)], [0] * (d // 2)
    qt, blocks = torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hkv, nb), dtype=torch.int32, device="cuda")
    o, lse = torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hq), device="cuda")
    ws_p, ws_a = e(aq.page_plan_workspace_bytes(B), torch.uint8), e(aq.kv4_sparse_workspace_bytes(T, Hq, Hkv, T, nb, d), torch.uint8)

    def step():
        aq.attnqat_page_plan(lens, want, table, T, free=(ring, state), workspace=ws_p, out=(lens, cu, slots, positions, state))
        aq.attnqat_kv_cache_append_rope(q, k, v, positions, rope, cache, slots, num_pages=num, out=qt)
        aq.attnqat_kv_summarize(cache, slots, summary, Hkv, d, num_pages=num)
        aq.attnqat_kv_select(qt, cu, summary, num, table, lens, Hkv, nb, max_q=T, out=blocks)
        aq.attnqat_fwd_kv4_sparse(qt, cu, cache, num, table, lens, Hkv, blocks, max_q=T, workspace=ws_a, out=(o, lse))

    hist = [np.zeros((2, 0, Hkv, d)) for _ in range(B)]
    h_lens, h_table, h_ring, h_state = np.zeros(B, int), table.cpu().numpy(), ring.cpu().numpy(), np.array([5, num, 0])
    # (the last step asks for 706 rows of 700: requests from the second on are refused, and keep what they had)
    wants = [[640, 1, 50, 0, 0], [641, 2, 56, 129, 400], [642, 3, 52, 700, 401], [760, 4, 53, 701, 900], [800, 5, 54, 702, 1000], [0, 6, 160, 900, 1001], [9, 700, 161, 901, 1002]]
    graph = None
    for i, w in enumerate(wants):
        x = S.bf16(rng.standard_normal((T, Hq + 2 * Hkv, d)))
        qkv.copy_(x.cuda())
        want.copy_(i32(w))
        if i == 3:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        h_lens, c, _, _, h_state = S.plan(h_lens, w, h_table, h_ring, h_state, T)
        for g, r in ((lens, h_lens), (cu, c), (table, h_table), (ring, h_ring), (state, h_state)):
            assert np.array_equal(g.cpu().numpy(), r), i
        assert np.array_equal(h_lens, w) == (i < 6) and h_state[2] == (4 if i == 6 else 0)
        w, tab = h_lens, h_table
        xd, turned_q = x.double().numpy(), qt.double().cpu().numpy()
        for b in range(B):
            n, old = c[b + 1] - c[b], hist[b].shape[1]
            rows = slice(c[b], c[b + 1])
            pos = (old + np.arange(n))[:, None]
            yq, size = P.turned(xd[rows, :Hq], pos, freqs, axis, "halves")
            assert (np.abs(turned_q[rows] - yq) <= 2.0 ** -8 * np.abs(yq) + 2.0 ** -21 * size).all()
            # (K: what the cache holds of it is phi of the turned rows, which the append's own test holds against the separate calls)
            turned_k = aq.attnqat_rope_fwd(k[rows].transpose(0, 1)[None], None, i32(pos), rope)[0][0].transpose(0, 1).double().cpu().numpy() if n else np.zeros((0, Hkv, d))
            new = [S.value(*S.phi(y)) for y in (turned_k, xd[rows, Hq + Hkv:])]
            hist[b] = np.concatenate([hist[b], np.stack(new)], axis=1)[:, :w[b]]      # (nothing of a request that was refused)
        host_cache, host_sum = cache.cpu().numpy().reshape(num, Hkv, 2, -1), summary.cpu().numpy()
        codes, scale = P.summary_parts(host_sum, Hkv, d)
        for b in range(B):
            if w[b]:
                kv = S.gather(host_cache, tab[b], w[b], Hkv, d)
                assert np.array_equal(kv[0], hist[b][0]) and np.array_equal(kv[1], hist[b][1])
            for p in tab[b, :w[b] // 128]:
                mc, ms = P.mean_of_page(host_cache, p, Hkv, d)
                assert np.array_equal(codes[p], mc) and np.array_equal(scale[p], ms)
        chosen = P.select(turned_q, c, codes, scale, tab, w, Hkv, nb, 1, 1, fill=0)
        live = c[-1]
        assert np.array_equal(blocks.cpu().numpy()[:live], chosen[:live])
        check_attention(o, lse, P.attend(turned_q, c, host_cache, tab, w, Hkv, chosen, d ** -0.5), i)


def test_binding_refuses(aq):
    q, cu, cache, num, table = attention_case([1, 2], [30, 20], 4, 2, 64, 1, tail=0)
    summary = torch.zeros(num * aq.kv_summary_page_bytes(2, 64), dtype=torch.uint8, device="cuda")
    good = dict(q=q.cuda(), cu_q=i32(cu), summary=summary, num_pages=num, page_table=dev(table), kv_lens=i32([30, 20]), Hkv=2, n_blocks=3)
    blocks = aq.attnqat_kv_select(**good)
    for kw in (dict(q=good["q"].float()), dict(q=good["q"].transpose(1, 2)), dict(q=q), dict(cu_q=i32([0, 1])), dict(kv_lens=good["kv_lens"].long()), dict(page_table=good["page_table"][:1]),
               dict(summary=summary[:-1]), dict(summary=summary.view(torch.int8)), dict(num_pages=num + 1), dict(num_pages=0), dict(Hkv=3), dict(n_blocks=0), dict(n_blocks=1025), dict(first=3),
               dict(last=0), dict(first=-1), dict(first=1 << 32), dict(last=(1 << 32) + 1), dict(out=blocks[:2]), dict(out=blocks.long()), dict(max_q=0)):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_kv_select(**{**good, **kw})
    good = dict(q=good["q"], cu_q=good["cu_q"], cache=dev(cache.reshape(-1)), num_pages=num, page_table=good["page_table"], kv_lens=good["kv_lens"], Hkv=2, blocks=blocks)
    aq.attnqat_fwd_kv4_sparse(**good)
    for kw in (dict(q=good["q"].float()), dict(blocks=blocks.long()), dict(blocks=blocks[:2]), dict(blocks=blocks[:, :1]), dict(blocks=blocks[..., :0]), dict(blocks=blocks.transpose(1, 2)),
               dict(cache=good["cache"][::2]), dict(num_pages=num + 1), dict(Hkv=3), dict(scale=0.0), dict(out=(good["q"], None)), dict(max_q=0),
               dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), dict(out=(torch.empty_like(good["q"]), torch.empty(3, 4, dtype=torch.float64, device="cuda")))):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_fwd_kv4_sparse(**{**good, **kw})
    slots = torch.arange(3, device="cuda")
    for args in ((good["cache"], slots.int(), summary, 2, 64), (good["cache"], slots, summary[:10], 2, 64), (good["cache"][:9], slots, summary, 2, 64), (good["cache"], slots, summary, 2, 32),
                 (good["cache"], slots[None], summary, 2, 64)):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_kv_summarize(*args)
