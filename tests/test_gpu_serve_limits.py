"""Serving steps at the ends of their ranges."""
import numpy as np
import pytest
import torch

from tests import serve_util as S
from tests.test_gpu_serve import _plan_case, attention_case, check_attention, dev, i32, run_attention

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


@pytest.mark.parametrize("kw", [dict(max_q=(1 << 32) + 1), dict(max_q=1 << 31), dict(window=(1 << 32) + 5), dict(window=1 << 31)])
def test_numbers_beyond_32_bits_are_not_cut(aq, kw):
    q, cu, cache, num_pages, table = attention_case([5, 60], [300, 200], 4, 2, 64, 1, tail=0)
    args = (q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([300, 200]), 2, True)
    o, lse = aq.attnqat_fwd_kv4_ragged(*args)
    out = torch.full_like(o, 5.0), torch.full_like(lse, 5.0)
    aq.attnqat_fwd_kv4_ragged(*args, **kw, out=out)
    assert torch.equal(out[0], o) and torch.equal(out[1], lse)
    for kw in (dict(max_q=1 - (1 << 32)), dict(window=5 - (1 << 32))):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_fwd_kv4_ragged(*args, **kw)


@pytest.mark.parametrize("n,kv,max_q", [([5, 2], [300, 20], 3), ([150, 40, 1], [400, 40, 9], 100), ([150, 97, 3], [150, 500, 9], 96), ([130, 300], [90, 700], 7)])
@pytest.mark.parametrize("G,causal", [(1, True), (2, True), (1, False)])
def test_sequences_cut_by_max_q(aq, n, kv, max_q, G, causal):
    """The first max_q rows of a sequence as if there were no others, the rest left alone."""
    q, cu, cache, num_pages, table = attention_case(n, kv, 2 * G, 2, 64, 1, tail=2)
    o, lse = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:2], 5.0, device="cuda")
    aq.attnqat_fwd_kv4_ragged(q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32(kv), 2, causal, max_q=max_q, out=(o, lse))
    m = np.minimum(n, max_q)
    rows = np.concatenate([cu[b] + np.arange(m[b]) for b in range(len(n))])
    ref = S.attend(q.double().numpy()[rows], np.concatenate([[0], np.cumsum(m)]), cache, table, kv, 2, causal, 0, 1.0 / 8.0)
    at = torch.from_numpy(rows).cuda()
    check_attention(o[at], lse[at], ref)
    o[at], lse[at] = 5.0, 5.0
    assert bool((o == 5.0).all()) and bool((lse == 5.0).all())


@pytest.mark.parametrize("n", [1, 3, 150])
@pytest.mark.parametrize("Hkv", [1, 3])
def test_sequences_far_apart(aq, n, Hkv):
    """Idle places, places of the other kernel and places without a key between sequences whose heads and pages do not divide evenly: each finds the next."""
    for B, at in ((700, (0, 65, 66, 130, 400, 699)), (1300, (3, 640, 1299)), (129, (0, 64, 128))):
        ns, kv = [0] * B, [0] * B
        for i, b in enumerate(at):
            ns[b], kv[b] = n, 200 + 77 * i
        for b in (1, 70, B - 2):                                  # of the other kernel, and with nothing to see
            ns[b], kv[b] = 120 if n == 1 else 1, 150
        ns[2], kv[2] = 110, 0
        run_attention(aq, ns, kv, 2 * Hkv, Hkv, 64, seed=B)


def test_idle_places_are_passed_by_in_no_time(aq):
    """Three prompts far apart among idle places of a step against the three alone.  One look at the lengths per place would be eight times their time; asked
    for 64 at once it is less than twice, most of it the sums over the lengths that every workgroup makes."""
    rng = np.random.default_rng(1)
    Hq, Hkv, d = 32, 8, 128
    kv, n = [3900, 4000, 4100], 700
    cache = dev(S.random_cache(33, Hkv, d, rng).reshape(-1))
    q = torch.randn(3 * n, Hq, d, device="cuda").bfloat16()
    times, outs = [], []
    for B in (3, 8192):
        lens, ns = np.zeros(B, int), np.zeros(B, int)
        lens[[0, B // 2, B - 1]], ns[[0, B // 2, B - 1]] = kv, n
        table = i32(np.tile(np.arange(33), (B, 1)))
        args = (q, i32(np.concatenate([[0], np.cumsum(ns)])), cache, 33, table, i32(lens), Hkv, True)
        ws = torch.empty(aq.kv4_ragged_workspace_bytes(3 * n, B, Hq, Hkv, n, 33, d), dtype=torch.uint8, device="cuda")
        t = []
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(4):
                out = aq.attnqat_fwd_kv4_ragged(*args, max_q=n, workspace=ws)
            end.record()
            end.synchronize()
            t.append(start.elapsed_time(end))
        times.append(min(t))
        outs.append(out)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert times[1] < 4 * times[0], times


def test_a_workspace_with_gaps_is_refused(aq):
    """What lies between its bytes is not the call's."""
    q, cu, cache, num_pages, table = attention_case([1, 2], [30, 20], 4, 2, 64, 1, tail=0)
    wide = torch.zeros((1 << 20, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(aq.AttnQatError):
        aq.attnqat_fwd_kv4_ragged(q.cuda(), i32(cu), dev(cache.reshape(-1)), num_pages, dev(table), i32([30, 20]), 2, True, workspace=wide[:, 0])
    with pytest.raises(aq.AttnQatError):
        aq.attnqat_page_plan(i32([1, 2]), i32([1, 3]), i32([[0], [1]]), 4, workspace=wide[:, 0])


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


@pytest.mark.parametrize("B,most,places,in_place", [(2, 3, 4, True), (60, 6, 150, False), (60, 6, 150, True), (900, 4, 700, False), (900, 4, 700, True), (1500, 3, 1000, True)])
def test_plan_with_a_ring_that_pages_given_back_do_not_fit(aq, B, most, places, in_place):
    """Pages come back into places that none of the free ones has; requests whose pages find none keep theirs and count as refused."""
    rng = np.random.default_rng(B)
    if B == 2:                                                   # one takes two of four free pages, the other has two to give: they would go where those are read
        old, want, table, T = np.array([0, 384]), np.array([256, 100]), np.array([[-1, -1, -1], [10, 11, 12]], np.int32), 300
        ring, state = np.arange(4, dtype=np.int32), np.array([3, 4])
    else:
        old, want, table, _, _, T = _plan_case(B, rng, most, 200, 1.0)
        ring, state = np.arange(10_000, 10_000 + places, dtype=np.int32), np.array([places - 5, places - 20])
    room, refused, kept = places - state[1], 0, want.copy()
    back = 0
    for b in range(B):                                           # the plan of requests that do not ask to give back what finds no place
        give = S.pages(int(old[b])) - S.pages(int(max(want[b], 0)))
        if give > 0:
            back += give
            if back > room:
                kept[b], refused = old[b], refused + 1
    assert refused > 0
    t_ref, r_ref = table.copy(), ring.copy()
    ref = S.plan(old, kept, t_ref, r_ref, state, T)
    ref[4][2] += refused
    lens, st, t_dev, r_dev = i32(old), i32(list(state) + [0]), dev(table), dev(ring)
    out = None
    if in_place:
        out = (lens, torch.empty(B + 1, dtype=torch.int32, device="cuda"), torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda"), st)
    got = aq.attnqat_page_plan(lens, i32(want), t_dev, T, free=(r_dev, st), out=out)
    for name, g, r in zip(("kv_lens", "cu_q", "slots", "positions", "free_state"), got, ref):
        assert np.array_equal(g.cpu().numpy(), r), name
    assert np.array_equal(t_dev.cpu().numpy(), t_ref) and np.array_equal(r_dev.cpu().numpy(), r_ref)
