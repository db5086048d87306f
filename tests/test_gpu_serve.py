"""A serving step over the NVFP4 cache: attnqat_page_plan, attnqat_kv_cache_append, attnqat_kv_cache_read and attnqat_fwd_kv4_ragged against
plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

from tests import serve_util as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------------ plan
def _plan_case(B, rng, most, grow, pool, T=None, head=None):
    """Requests that grow, stay, shrink or end; a ring that starts anywhere."""
    old = rng.integers(0, most * 128 + 1, B)
    kind = rng.random(B)
    want = np.where(kind < 0.6, old + rng.integers(0, grow + 1, B), np.where(kind < 0.8, old - rng.integers(0, 300, B), np.where(kind < 0.9, old, 0)))
    held = sum(S.pages(int(o)) for o in old)
    need = int(sum(max(0, S.pages(int(max(w, 0))) - S.pages(int(o))) for o, w in zip(old, want)))
    free = int(need * pool) + 1
    num = held + max(free, need) + 1
    order = rng.permutation(num).astype(np.int32)
    table = np.full((B, most), -1, np.int32)
    at = 0
    for b in range(B):
        n = S.pages(int(old[b]))
        table[b, :n] = order[at:at + n]
        at += n
    head = int(rng.integers(0, num)) if head is None else head
    ring = np.full(num, -1, np.int32)
    ring[(head + np.arange(free)) % num] = order[at:at + free] if at + free <= num else 0
    T = int(np.clip(want - old, 0, None).sum()) + 3 if T is None else T
    return old, want, table, ring, np.array([head, free]), T


def _check_plan(aq, old, want, table, ring, state, T, ws=None):
    t_dev, r_dev = dev(table), None if ring is None else dev(ring)
    free = None if ring is None else (r_dev, i32(state))
    got = aq.attnqat_page_plan(i32(old), i32(want), t_dev, T, free=free, workspace=ws)
    t_ref, r_ref = table.copy(), None if ring is None else ring.copy()
    ref = S.plan(old, want, t_ref, r_ref, state, T)
    for name, g, r in zip(("kv_lens", "cu_q", "slots", "positions", "free_state"), got, ref):
        if r is not None:
            assert np.array_equal(g.cpu().numpy(), r), name
    assert np.array_equal(t_dev.cpu().numpy(), t_ref)
    if ring is not None:
        assert np.array_equal(r_dev.cpu().numpy(), r_ref)


@pytest.mark.parametrize("B,most,grow,pool", [(1, 1, 1, 1.0), (1, 300, 40000, 1.0), (7, 3, 1, 1.0), (64, 5, 200, 0.5), (257, 9, 1, 0.7), (1023, 4, 40, 0.9),
                                              (1025, 4, 600, 0.3), (3001, 2, 130, 0.5)])
def test_plan(aq, B, most, grow, pool):
    rng = np.random.default_rng(B + most)
    _check_plan(aq, *_plan_case(B, rng, most, grow, pool))


@pytest.mark.parametrize("T", [0, 1, 255, 256, 257, 4000])
def test_plan_of_less_capacity_than_asked_for(aq, T):
    rng = np.random.default_rng(T)
    old, want, table, ring, state, _ = _plan_case(50, rng, 6, 300, 1.0)
    _check_plan(aq, old, want, table, ring, state, T)


def test_plan_without_a_ring_and_with_holes_in_the_table(aq):
    rng = np.random.default_rng(5)
    old, want, table, _, _, T = _plan_case(40, rng, 6, 300, 1.0)
    table[:] = rng.integers(-2, 1000, table.shape)
    _check_plan(aq, old, want, table, None, None, T)


def test_plan_of_lengths_out_of_range(aq):
    table = np.arange(12, dtype=np.int32).reshape(4, 3)
    _check_plan(aq, [-5, 384, 10_000, 100], [3, 385, 20, -7], table, np.arange(20, 30, dtype=np.int32), [9, 4], 64)


def test_plan_ring_wraps_and_pages_come_back(aq):
    """Many steps in place: no page is lost or owned twice."""
    rng = np.random.default_rng(11)
    B, most, num = 20, 8, 70
    lens, table = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B, most), -1, dtype=torch.int32, device="cuda")
    ring, state = i32(rng.permutation(num)), i32([37, num, 0])
    h_lens, h_table, h_ring, h_state = np.zeros(B, int), np.full((B, most), -1, np.int32), ring.cpu().numpy(), np.array([37, num, 0])
    cu, slots, positions = torch.empty(B + 1, dtype=torch.int32, device="cuda"), torch.empty(4096, dtype=torch.int64, device="cuda"), torch.empty(4096, dtype=torch.int32, device="cuda")
    for step in range(25):
        want = np.where(rng.random(B) < 0.2, 0, np.clip(h_lens + rng.integers(-200, 500, B), 0, most * 128))
        aq.attnqat_page_plan(lens, i32(want), table, 4096, free=(ring, state), out=(lens, cu, slots, positions, state))
        h_lens, h_cu, h_slots, h_pos, h_state = S.plan(h_lens, want, h_table, h_ring, h_state, 4096)
        for g, r in ((lens, h_lens), (cu, h_cu), (slots, h_slots), (positions, h_pos), (state, h_state), (table, h_table), (ring, h_ring)):
            assert np.array_equal(g.cpu().numpy(), r), step
        held = [int(h_table[b, i]) for b in range(B) for i in range(S.pages(int(h_lens[b])))]
        free = [int(h_ring[(h_state[0] + i) % num]) for i in range(h_state[1])]
        assert sorted(held + free) == list(range(num))


# ------------------------------------------------------------------------------------------------------------ append, read
def _slots(T, num_pages, rng, bad=0.1):
    s = rng.permutation(num_pages * 128)[:T].astype(np.int64)
    if T > 2:
        out = rng.random(T) < bad
        s[out] = rng.choice([-1, -(1 << 40), num_pages * 128, 1 << 40], out.sum())
    return s


def _views(x, layout):
    """x [T, heads, d] on the GPU in another layout, same values."""
    T, H, d = x.shape
    if layout == "plain":
        return x.contiguous()
    if layout == "fused":                                        # a piece of a projection's output
        y = torch.full((T, H + 3, d), float("nan"), dtype=x.dtype, device="cuda")
        y[:, 1:1 + H] = x
        return y[:, 1:1 + H]
    y = torch.full((H, T + 2, d + 8), float("nan"), dtype=x.dtype, device="cuda")          # heads outermost, padded
    y[:, 1:1 + T, :d] = x.transpose(0, 1)
    return y[:, 1:1 + T, :d].transpose(0, 1)


@pytest.mark.parametrize("layout", ["plain", "fused", "heads"])
@pytest.mark.parametrize("T,Hkv,d", [(1, 1, 64), (1, 8, 128), (31, 3, 128), (33, 2, 64), (130, 1, 128), (1000, 5, 64)])
def test_append_and_read(aq, T, Hkv, d, layout):
    rng = np.random.default_rng(T + Hkv)
    num_pages = S.pages(T) + 2
    cache0 = rng.integers(0, 256, num_pages * aq.kv_cache_page_bytes_nvfp4(Hkv, d), dtype=np.uint8)
    slots = _slots(T, num_pages, rng)
    x = rng.standard_normal((2, T, Hkv, d)) * np.exp2(rng.integers(-14, 8, (2, T, Hkv, d // 16))).repeat(16, -1)
    x[0, 0, 0, :16] = 0.0
    x[1, -1, -1, 16:32] = 1e-30
    x[1, 0, 0, 3] = 3e38                                         # saturates its block's scale
    xb = S.bf16(x)
    cache = dev(cache0)
    k, v = (_views(xb[i].cuda(), layout) for i in range(2))
    aq.attnqat_kv_cache_append(k, v, cache, dev(slots))
    ref = cache0.copy().reshape(num_pages, Hkv, 2, -1)
    n = 128 * d // 2
    ref_c, ref_s = ref[..., :n].reshape(num_pages, Hkv, 2, 128, d // 2).copy(), ref[..., n:].reshape(num_pages, Hkv, 2, 128, d // 16).copy()
    inside = (slots >= 0) & (slots < num_pages * 128)
    values = np.zeros((2, T, Hkv, d))
    for i in range(2):
        c, s = S.phi(xb[i].double().numpy())
        pg, off = slots[inside] // 128, slots[inside] % 128
        ref_c[pg, :, i, off], ref_s[pg, :, i, off] = c[inside], s[inside]
        values[i][inside] = S.value(c, s)[inside]
    got_c, got_s = S.parts(cache.cpu().numpy(), Hkv, d)
    assert np.array_equal(got_s, ref_s)                          # (every other byte of the cache as it was)
    assert np.array_equal(got_c, ref_c)
    out = None if layout == "plain" else tuple(_views(torch.zeros((T, Hkv, d), dtype=torch.bfloat16, device="cuda"), layout) for _ in range(2))
    kr, vr = aq.attnqat_kv_cache_read(cache, dev(slots), Hkv, d, out=out)
    assert np.array_equal(kr.double().cpu().numpy(), values[0]) and np.array_equal(vr.double().cpu().numpy(), values[1])


def test_read_leaves_what_lies_between_rows(aq):
    rng = np.random.default_rng(3)
    cache = dev(S.random_cache(2, 2, 64, rng).reshape(-1))
    buf = torch.full((9, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    aq.attnqat_kv_cache_read(cache, dev(np.arange(9, dtype=np.int64)), 2, 64, out=(buf[:, 0:2], buf[:, 2:4]))
    assert bool((buf[:, 4] == 7.0).all()) and not bool((buf[:, :4] == 7.0).all())


def test_append_agrees_with_the_write_of_one_sequence(aq):
    rng = np.random.default_rng(4)
    n, Hkv, d = 300, 4, 128
    x = S.bf16(rng.standard_normal((2, n, Hkv, d))).cuda()
    ids = i32([3, 0, 2])
    a, b = (torch.zeros(4 * aq.kv_cache_page_bytes_nvfp4(Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    aq.attnqat_kv_cache_write(x[0].transpose(0, 1)[None].contiguous(), x[1].transpose(0, 1)[None].contiguous(), a, ids)
    pos = torch.arange(n, device="cuda")
    aq.attnqat_kv_cache_append(x[0], x[1], b, ids[pos // 128].long() * 128 + pos % 128)
    assert torch.equal(a, b)


def test_empty_steps(aq):
    cache = torch.zeros(aq.kv_cache_page_bytes_nvfp4(2, 64), dtype=torch.uint8, device="cuda")
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.empty(0, dtype=torch.int64, device="cuda")
    aq.attnqat_kv_cache_append(none, none, cache, slots)
    k, v = aq.attnqat_kv_cache_read(cache, slots, 2, 64)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)
    o, lse = aq.attnqat_fwd_kv4_ragged(none, i32([0, 0]), cache, 1, i32([[0]]), i32([5]), 2, True)
    assert o.shape == (0, 2, 64) and lse.shape == (0, 2)


# ------------------------------------------------------------------------------------------------------------ attention
def check_attention(o, lse, ref, what=""):
    """Against 64 bits.  o: rounded to bf16 (half a step: 2^-9 of the value, 2^-8 where the fp32 value lies across a power of two), the
    probabilities rounded to fp16 (each by a relative 2^-12, below 2^-14 of the largest by 2^-25 of it: together at most 2^-12 sum p |v| and what
    a row's smallest probabilities add), scores with a few fp32 roundings: an error e of an exponent is a relative e of a probability.  Scores here are
    below 2^7, dot products of fp32 terms: e <= 2^-14.  So |error| <= 2^-8 |o| + 2^-10.5 sum p |v|.  lse: e, and the logarithm's own rounding."""
    ro, rl, wt = ref
    have = ~np.isnan(rl)
    go, gl = o.double().cpu().numpy(), lse.double().cpu().numpy()
    err = np.abs(go - ro)[have] - (2.0 ** -8 * np.abs(ro) + 2.0 ** -10.5 * wt)[have]
    assert not np.isnan(go[have]).any(), what
    assert err.max(initial=0.0) <= 0.0, (what, float(err.max()))
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(gl)[have], empty[have]), what
    fin = have & ~empty
    assert np.abs(gl - np.where(fin, rl, 0.0))[fin].max(initial=0.0) <= 2.0 ** -14 + 2.0 ** -22 * np.abs(rl[fin]).max(initial=0.0), what


def attention_case(n, kv, Hq, Hkv, d, seed, tail=0, q_scale=1.0):
    rng = np.random.default_rng(seed)
    table, num_pages = S.make_table(kv, rng)
    cache = S.random_cache(num_pages, Hkv, d, rng)
    # K so that scores are a few units: scale bytes of K lower; slots behind a sequence's end full of stale bytes, NaN scales among them
    codes, scales = cache[..., :64 * d], cache[..., 64 * d:]
    scales[:, :, 0] = np.clip(scales[:, :, 0].astype(int) - 16, 8, None)
    for b, length in enumerate(kv):
        if length % 128:
            p = table[b, length // 128]
            for i in range(2):
                scales[p, :, i].reshape(Hkv, 128, d // 16)[:, length % 128:] = rng.choice([127, 255, 126], (Hkv, 128 - length % 128, d // 16))
    cu = np.concatenate([[0], np.cumsum(n)])
    q = S.bf16(rng.standard_normal((int(cu[-1]) + tail, Hq, d)) * q_scale)
    return q, cu, cache, num_pages, table


def run_attention(aq, n, kv, Hq, Hkv, d, causal=True, window=0, scale=None, seed=0, tail=3, layout="plain", max_q=None, q_scale=1.0, ws=None):
    q, cu, cache, num_pages, table = attention_case(n, kv, Hq, Hkv, d, seed, tail, q_scale)
    T = q.shape[0]
    qd = _views(q.cuda(), layout)
    o = _views(torch.full((T, Hq, d), 5.0, dtype=torch.bfloat16, device="cuda"), layout)
    lse = torch.full((T, Hq), 5.0, device="cuda")
    aq.attnqat_fwd_kv4_ragged(qd, i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32(kv), Hkv, causal, max_q=max_q or max(max(n), 1), window=window,
                              scale=scale, workspace=ws, out=(o, lse))
    ref = S.attend(q.double().numpy(), cu, cache, table, kv, Hkv, causal, window, 1.0 / np.sqrt(d) if scale is None else scale)
    check_attention(o, lse, ref, (n, kv, Hq, Hkv, d))
    if tail:                                                     # rows behind the last sequence: left as they were
        assert bool((o[-tail:] == 5.0).all()) and bool((lse[-tail:] == 5.0).all())
    return o, lse


@pytest.mark.parametrize("kv", [[1], [2], [31], [32], [33], [63], [64], [65], [127], [128], [129], [255], [257], [1000], [4097], [1, 128, 5, 640, 33]])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 128), (4, 4, 64)])
def test_one_query(aq, kv, Hq, Hkv, d):
    run_attention(aq, [1] * len(kv), kv, Hq, Hkv, d, seed=len(kv) + kv[0])


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 15, 16, 17, 32, 33, 71])
def test_heads_of_a_group(aq, G):
    run_attention(aq, [1, 1], [300, 77], 2 * G, 2, 64 if G % 2 else 128, seed=G)


@pytest.mark.parametrize("n,kv", [([1, 7, 3, 16, 2], [1, 7, 500, 16, 131]), ([5, 100, 1], [5, 100, 1]), ([129, 1, 64], [129, 400, 700]), ([300], [1111]),
                                  ([0, 4, 0, 0, 9, 0], [50, 60, 0, 128, 9, 3]), ([260, 3], [300, 3])])
@pytest.mark.parametrize("Hq,Hkv,d,causal,window", [(8, 2, 128, True, 0), (6, 2, 64, True, 40), (4, 4, 128, False, 0), (8, 1, 128, True, 1)])
def test_ragged(aq, n, kv, Hq, Hkv, d, causal, window):
    run_attention(aq, n, kv, Hq, Hkv, d, causal, window, seed=sum(n))


@pytest.mark.parametrize("window", [1, 2, 31, 127, 128, 129, 200, 511, 5000])
def test_window(aq, window):
    run_attention(aq, [1, 5, 130, 1], [900, 640, 700, 40], 4, 1, 64, window=window, seed=window)
    run_attention(aq, [1, 3], [2000, 129], 8, 2, 128, window=window, seed=window)


def test_more_queries_than_keys(aq):
    """Rows in front of the sequence's first position see nothing: o = 0, lse = -inf; so does every row of a sequence without keys."""
    for causal in (True, False):
        run_attention(aq, [10, 3, 40, 200], [4, 0, 0, 150], 4, 2, 128, causal, seed=8)
        run_attention(aq, [10, 3, 40, 200], [4, 0, 0, 150], 4, 2, 64, causal, seed=9)


@pytest.mark.parametrize("layout", ["fused", "heads"])
def test_strided_rows(aq, layout):
    run_attention(aq, [1, 9, 40], [200, 300, 40], 6, 3, 128, layout=layout, seed=3)
    run_attention(aq, [1], [200], 1, 1, 64, layout=layout, seed=3, tail=0)


@pytest.mark.parametrize("layout", ["plain", "fused", "heads"])
@pytest.mark.parametrize("Hq,Hkv,d", [(6, 2, 128), (10, 2, 64), (1, 1, 128), (7, 1, 64)])
def test_strided_rows_of_long_pieces(aq, layout, Hq, Hkv, d):
    """Row tiles that end inside a wave's rows, in a query's heads and at one row; nothing written between rows or behind them."""
    for n, kv in (([301, 1, 97], [301, 40, 500]), ([257], [257])):
        q, cu, cache, num_pages, table = attention_case(n, kv, Hq, Hkv, d, 11, tail=2)
        T = q.shape[0]
        whole = torch.full((T, Hq + 3, d), 7.0, dtype=torch.bfloat16, device="cuda")
        o = whole[:, 1:Hq + 1] if layout == "fused" else torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        if layout == "heads":
            whole = torch.full((Hq, T + 5, d), 7.0, dtype=torch.bfloat16, device="cuda")
            o = whole[:, 2:T + 2].transpose(0, 1)
        lse = torch.full((T, Hq), 7.0, device="cuda")
        aq.attnqat_fwd_kv4_ragged(_views(q.cuda(), layout), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32(kv), Hkv, True, max_q=max(n), out=(o, lse))
        check_attention(o, lse, S.attend(q.double().numpy(), cu, cache, table, kv, Hkv, True, 0, 1.0 / np.sqrt(d)), (layout, n, Hq, Hkv, d))
        assert bool((o[-2:] == 7.0).all()) and bool((lse[-2:] == 7.0).all())
        if layout == "fused":
            assert bool((whole[:, 0] == 7.0).all()) and bool((whole[:, Hq + 1:] == 7.0).all())
        if layout == "heads":
            assert bool((whole[:, :2] == 7.0).all()) and bool((whole[:, T + 2:] == 7.0).all())


@pytest.mark.parametrize("scale", [0.01, 0.5])
def test_scale(aq, scale):
    run_attention(aq, [1, 20], [200, 300], 4, 2, 64, scale=scale, seed=3, q_scale=0.25)


@pytest.mark.parametrize("q_scale", [1e-38, 1e-20, 1e30])
def test_queries_far_from_one(aq, q_scale):
    """Large ones are brought back by the factor of the scores, small ones give even probabilities."""
    run_attention(aq, [1, 20], [200, 300], 4, 2, 128, scale=1e-31 if q_scale > 1 else None, seed=3, q_scale=q_scale)


@pytest.mark.parametrize("scale", [1e-44, 1e-20, None])
@pytest.mark.parametrize("causal", [True, False])
def test_queries_of_zeros_and_least_factors(aq, scale, causal):
    """Even probabilities over the keys that a row sees: the factor of the scores may lie below the least number, masked keys stay masked."""
    for n, kv in (([1, 20], [200, 300]), ([70, 90], [200, 90])):
        for q_scale in (0.0, 1e-3):
            run_attention(aq, n, kv, 4, 2, 128, causal, scale=scale, seed=3, q_scale=q_scale)
            run_attention(aq, n, kv, 4, 2, 64, causal, scale=scale, seed=3, q_scale=q_scale)


def test_nan_stays_in_its_row(aq):
    for n, G in (([1, 3], 4), ([60, 40], 2)):
        q, cu, cache, num_pages, table = attention_case(n, [300, 200], 2 * G, 2, 128, 1, tail=0)
        args = (i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([300, 200]), 2, True)
        qd = q.cuda()
        o, lse = aq.attnqat_fwd_kv4_ragged(qd, *args)
        qn = qd.clone()
        qn[1, 3, 17] = float("nan")
        on, ln = aq.attnqat_fwd_kv4_ragged(qn, *args)
        assert bool(on[1, 3].isnan().all()) and bool(ln[1, 3].isnan())
        on[1, 3], ln[1, 3] = o[1, 3], lse[1, 3]
        assert torch.equal(on, o) and torch.equal(ln, lse)


def test_rows_beyond_max_q_are_left_out(aq):
    q, cu, cache, num_pages, table = attention_case([5, 2], [300, 20], 4, 2, 64, 1)
    o, lse = torch.full((7, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((7, 4), 5.0, device="cuda")
    args = (q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([300, 20]), 2, True)
    aq.attnqat_fwd_kv4_ragged(*args, max_q=3, out=(o, lse))
    torch.cuda.synchronize()
    assert bool((o[3:5] == 5.0).all()) and bool((lse[3:5] == 5.0).all()) and not bool((o[:3] == 5.0).all()) and not bool((o[5:] == 5.0).all())


def test_pages_outside_the_cache_read_as_zeros(aq):
    q, cu, cache, num_pages, table = attention_case([1, 20], [700, 300], 4, 2, 128, 2)
    table[0, 2], table[1, 0], table[0, 4] = -1, num_pages, 1 << 30
    o, lse = aq.attnqat_fwd_kv4_ragged(q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([700, 300]), 2, True)
    check_attention(o, lse, S.attend(q.double().numpy(), cu, cache, table, [700, 300], 2, True, 0, 128 ** -0.5))


def test_without_lse_and_defaults(aq):
    q, cu, cache, num_pages, table = attention_case([1, 20], [700, 300], 4, 2, 128, 2)
    args = (q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([700, 300]), 2, True)
    o, lse = aq.attnqat_fwd_kv4_ragged(*args)
    o2 = torch.empty_like(o)
    aq.attnqat_fwd_kv4_ragged(*args, out=(o2, None))
    assert torch.equal(o, o2)


# ------------------------------------------------------------------------------------------------------------ together
def test_steps_of_a_server(aq):
    """Plan, append, attend, step after step: prompts in pieces, single tokens, drafted tokens taken back, requests that end.  Every step against
    attention over the values of what was appended; and once as a captured graph whose lengths change between replays."""
    rng = np.random.default_rng(21)
    B, Hq, Hkv, d, most, num, T = 6, 8, 2, 128, 6, 24, 400
    e = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    lens, want, table, ring, state = e(B), e(B), torch.full((B, most), -1, dtype=torch.int32, device="cuda"), i32(rng.permutation(num)), i32([5, num, 0])
    cu, slots, positions = e(B + 1), e(T, torch.int64), e(T)
    cache = dev(rng.integers(0, 256, num * aq.kv_cache_page_bytes_nvfp4(Hkv, d), dtype=np.uint8))
    qkv = torch.zeros((T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=1)
    o, lse = torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hq), device="cuda")
    ws_p = e(aq.page_plan_workspace_bytes(B), torch.uint8)
    ws_a = e(aq.kv4_ragged_workspace_bytes(T, B, Hq, Hkv, T, most, d), torch.uint8)

    def step():
        aq.attnqat_page_plan(lens, want, table, T, free=(ring, state), workspace=ws_p, out=(lens, cu, slots, positions, state))
        aq.attnqat_kv_cache_append(k, v, cache, slots, num_pages=num)
        aq.attnqat_fwd_kv4_ragged(q, cu, cache, num, table, lens, Hkv, True, max_q=T, workspace=ws_a, out=(o, lse))

    hist = [np.zeros((2, 0, Hkv, d)) for _ in range(B)]
    wants = [[130, 1, 50, 0, 0, 200], [131, 2, 56, 129, 0, 201], [132, 3, 52, 130, 300, 202], [0, 4, 53, 131, 301, 203], [7, 5, 54, 400, 302, 0], [8, 6, 160, 0, 303, 90],
             [9, 7, 161, 128, 300, 91]]
    graph = None
    for i, w in enumerate(wants):
        x = S.bf16(rng.standard_normal((T, Hq + 2 * Hkv, d)))
        qkv.copy_(x.cuda())
        want.copy_(i32(w))
        if i == 3:                                               # (an eager run first; capturing enqueues nothing)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        got_lens, got_cu = lens.cpu().numpy(), cu.cpu().numpy()
        assert np.array_equal(got_lens, w) and int(state[2]) == 0
        xd = x.double().numpy()
        for b in range(B):
            n, old = got_cu[b + 1] - got_cu[b], hist[b].shape[1]
            assert n == max(0, w[b] - old)
            new = [S.value(*S.phi(xd[got_cu[b]:got_cu[b + 1], Hq + j * Hkv:Hq + (j + 1) * Hkv])) for j in range(2)]
            hist[b] = np.concatenate([hist[b], np.stack(new)], axis=1)[:, :w[b]]
        # the reference on a cache of its own, laid out page by page
        refs = np.zeros((B, most * 128, 2, Hkv, d))
        for b in range(B):
            refs[b, :w[b]] = hist[b].transpose(1, 0, 2, 3)
        kv, vv = aq.attnqat_kv_cache_read(cache, dev(np.concatenate([table.cpu().numpy()[b, np.arange(w[b]) // 128].astype(np.int64) * 128 + np.arange(w[b]) % 128
                                                                     for b in range(B)])), Hkv, d, num_pages=num)
        assert np.array_equal(kv.double().cpu().numpy(), np.concatenate([refs[b, :w[b], 0] for b in range(B)]))
        assert np.array_equal(vv.double().cpu().numpy(), np.concatenate([refs[b, :w[b], 1] for b in range(B)]))
        host_cache = cache.cpu().numpy().reshape(num, Hkv, 2, -1)
        check_attention(o, lse, S.attend(xd[:, :Hq], got_cu, host_cache, table.cpu().numpy(), w, Hkv, True, 0, d ** -0.5), i)


def test_binding_refuses(aq):
    """Tensors that do not fit what the call is told (checked before the library is called)."""
    q, cu, cache, num_pages, table = attention_case([1, 2], [30, 20], 4, 2, 64, 1, tail=0)
    good = dict(q=q.cuda(), cu_q=i32(cu), cache=dev(cache.reshape(-1)), num_pages=num_pages, page_table=dev(table), kv_lens=i32([30, 20]), Hkv=2, causal=True)
    aq.attnqat_fwd_kv4_ragged(**good)
    bad = [dict(q=good["q"].float()), dict(q=good["q"].transpose(1, 2)), dict(q=q), dict(cu_q=i32([0, 1])), dict(cu_q=good["cu_q"].long()), dict(kv_lens=good["kv_lens"].cpu()),
           dict(page_table=good["page_table"][:1]), dict(page_table=good["page_table"].t()), dict(num_pages=num_pages + 1), dict(num_pages=0), dict(cache=good["cache"].view(torch.int8)),
           dict(cache=good["cache"][::2]), dict(Hkv=3), dict(window=3, causal=False), dict(scale=-1.0), dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
           dict(out=(torch.empty_like(good["q"]), torch.empty(3, 4, dtype=torch.float64, device="cuda"))), dict(out=(good["q"], None)), dict(max_q=0)]
    for kw in bad:
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_fwd_kv4_ragged(**{**good, **kw})
    k, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.arange(3, device="cuda")
    for args in ((k, k[:2], good["cache"], slots), (k, k, good["cache"], slots[:2]), (k, k, good["cache"], slots.int()), (k, k.half(), good["cache"], slots), (k, k, good["cache"][:100], slots)):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_kv_cache_append(*args)
    for args in ((good["cache"], slots.int(), 2, 64), (good["cache"], slots, 2, 32), (good["cache"][:9], slots, 2, 64)):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_kv_cache_read(*args)
    lens = i32([1, 2])
    for args in ((lens, i32([1]), i32([[0], [1]]), 4), (lens, lens.long(), i32([[0], [1]]), 4), (lens, lens, i32([0, 1]), 4), (lens, lens, i32([[0], [1]]), -1),
                 (lens, lens, i32([[0], [1]]), 4, (i32([0]), i32([0])))):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_page_plan(*args)


@pytest.mark.parametrize("B,T", [(30, 4096), (30, 4097), (1024, 6000), (1025, 6000), (200, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_in_place_and_beside(aq, B, T, in_place):
    """The results do not depend on where they go, whichever launches the sizes take."""
    rng = np.random.default_rng(B + T)
    old, want, table, ring, state, _ = _plan_case(B, rng, 40, 2 * T // B, 0.9)
    t_ref, r_ref = table.copy(), ring.copy()
    ref = S.plan(old, want, t_ref, r_ref, state, T)
    lens, st, t_dev, r_dev = i32(old), i32(list(state) + [7]), dev(table), dev(ring)
    out = None
    if in_place:
        out = (lens, torch.empty(B + 1, dtype=torch.int32, device="cuda"), torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda"), st)
    got = aq.attnqat_page_plan(lens, i32(want), t_dev, T, free=(r_dev, st), out=out)
    for g, r in zip(got, ref):
        assert np.array_equal(g.cpu().numpy(), r)
    assert np.array_equal(t_dev.cpu().numpy(), t_ref) and np.array_equal(r_dev.cpu().numpy(), r_ref)
    if not in_place:
        assert np.array_equal(lens.cpu().numpy(), old) and np.array_equal(st.cpu().numpy()[:2], state)


def test_many_sequences(aq):
    """More sequences than a workgroup has threads, some of them with enough rows for the kernel of many, some empty."""
    rng = np.random.default_rng(31)
    for B in (300, 700):
        kv = [int(x) for x in rng.integers(0, 260, B)]
        n = [min(k, int(rng.choice([0, 1, 1, 1, 2]))) for k in kv]
        for b in (3, B // 2, B - 1):
            kv[b], n[b] = 200, 150
        run_attention(aq, n, kv, 2, 1, 64, seed=B)


@pytest.mark.parametrize("n,kv", [([1], [20000]), ([1, 5], [9000, 17001]), ([150], [17001]), ([60, 1], [8193, 16385])])
@pytest.mark.parametrize("window", [0, 9000])
def test_long_sequences(aq, n, kv, window):
    """More pages than a wave has lanes."""
    run_attention(aq, n, kv, 4, 1, 64, window=window, seed=kv[0])


def test_offsets_beyond_32_bits(aq):
    Hkv, d = 8, 128
    page = aq.kv_cache_page_bytes_nvfp4(Hkv, d)
    num = (5 << 30) // page
    cache = torch.zeros(num * page, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(6)
    kv, n = [200, 150], [1, 60]
    table = np.array([[num - 1, 3], [num - 2, num - 3]], np.int32)
    pos = [np.arange(k) for k in kv]
    slots = np.concatenate([table[b, p // 128].astype(np.int64) * 128 + p % 128 for b, p in enumerate(pos)])
    x = S.bf16(rng.standard_normal((2, sum(kv), Hkv, d)))
    aq.attnqat_kv_cache_append(x[0].cuda(), x[1].cuda(), cache, dev(slots))
    k, v = aq.attnqat_kv_cache_read(cache, dev(slots), Hkv, d)
    want = [S.value(*S.phi(x[i].double().numpy())) for i in range(2)]
    assert np.array_equal(k.double().cpu().numpy(), want[0]) and np.array_equal(v.double().cpu().numpy(), want[1])
    q = S.bf16(rng.standard_normal((61, 16, d)))
    o, lse = aq.attnqat_fwd_kv4_ragged(q.cuda(), i32([0, 1, 61]), cache, num, dev(table), i32(kv), Hkv, True)
    used = sorted(set(table.reshape(-1)))
    small = cache.view(num, -1)[torch.tensor(used, device="cuda")].cpu().numpy().reshape(len(used), Hkv, 2, -1)      # the reference: those pages alone
    table_s = np.array([[used.index(t) for t in row] for row in table], np.int32)
    check_attention(o, lse, S.attend(q.double().numpy(), [0, 1, 61], small, table_s, kv, Hkv, True, 0, d ** -0.5))


def test_nothing_to_do_leaves_the_outputs(aq):
    q, cu, cache, num_pages, table = attention_case([3, 2], [30, 20], 4, 2, 64, 1, tail=0)
    o, lse = torch.full((5, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 4), 5.0, device="cuda")
    aq.attnqat_fwd_kv4_ragged(q.cuda(), i32([0, 0, 0]), dev(cache.reshape(-1)), num_pages, dev(table), i32([30, 20]), 2, True, out=(o, lse))
    assert bool((o == 5.0).all()) and bool((lse == 5.0).all())


def test_offsets_out_of_order_stay_inside(aq):
    """cu_q that does not rise or leaves [0, T], lengths beyond the table: clamped, nothing outside the tensors is touched."""
    q, cu, cache, num_pages, table = attention_case([3, 2, 4], [30, 20, 128], 4, 2, 64, 1, tail=0)
    for c, lens in (([-5, 4, 2, 400], [30, 20, 128]), ([0, 3, 5, 9], [-7, 1 << 30, 1 << 20])):
        o = torch.full((11, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        aq.attnqat_fwd_kv4_ragged(q.cuda(), i32(c), dev(cache.reshape(-1)), num_pages, dev(np.clip(table, 0, num_pages - 1)), i32(lens), 2, True, out=(o[1:10], None))
        torch.cuda.synchronize()
        assert bool((o[0] == 5.0).all()) and bool((o[10] == 5.0).all())


@pytest.mark.parametrize("n,kv,window", [([1, 1, 4], [3000, 40, 900], 0), ([300, 1, 20], [700, 500, 60], 0), ([300, 1, 20], [700, 500, 60], 64)])
def test_same_bits_again_on_another_stream_and_in_a_graph(aq, n, kv, window):
    q, cu, cache, num_pages, table = attention_case(n, kv, 8, 2, 128, 5, tail=0)
    args = (q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32(kv), 2, True)
    ws = torch.empty(aq.kv4_ragged_workspace_bytes(q.shape[0], len(n), 8, 2, max(n), table.shape[1], 128), dtype=torch.uint8, device="cuda")
    o, lse = aq.attnqat_fwd_kv4_ragged(*args, max_q=max(n), window=window)
    ws.random_(0, 256)                                           # (what lies in the workspace does not matter)
    out = tuple(torch.empty_like(t) for t in (o, lse))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aq.attnqat_fwd_kv4_ragged(*args, max_q=max(n), window=window, workspace=ws, out=out)
    side.synchronize()
    assert torch.equal(out[0], o) and torch.equal(out[1], lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        aq.attnqat_fwd_kv4_ragged(*args, max_q=max(n), window=window, workspace=ws, out=out)
    for _ in range(3):
        out[0].zero_(), out[1].zero_(), ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], o) and torch.equal(out[1], lse)


def test_one_row_of_a_batch_does_not_depend_on_padding_rows(aq):
    """A step captured for more rows than it has: same results as without the rows behind."""
    q, cu, cache, num_pages, table = attention_case([1, 2], [300, 200], 4, 2, 128, 5, tail=30)
    args = (i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([300, 200]), 2, True)
    o, lse = aq.attnqat_fwd_kv4_ragged(q.cuda(), *args, max_q=2)
    o3, lse3 = aq.attnqat_fwd_kv4_ragged(q[:3].cuda(), *args, max_q=2)
    assert torch.equal(o[:3], o3) and torch.equal(lse[:3], lse3)
