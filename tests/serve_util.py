"""References of the serving step's operators (64 bits, numpy, sequence by sequence) and caches to run them on."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1 = np.concatenate([GRID, -GRID])
E4M3 = np.array([np.nan if i & 127 == 127 else (-1.0) ** (i >> 7) * ((i & 7) * 2.0 ** -9 if (i >> 3) & 15 == 0 else (8 + (i & 7)) * 2.0 ** (((i >> 3) & 15) - 10))
                 for i in range(256)])
PAGE = 128


def pages(n):
    return (n + PAGE - 1) // PAGE


def plan(old, want, table, ring, state, T):
    """attnqat_page_plan, request after request; table and ring are changed in place.  ring None: the table is complete."""
    most, cap = table.shape[1], 0 if ring is None else len(ring)
    head, count = (0, 0) if ring is None else (min(max(int(state[0]), 0), cap - 1), min(max(int(state[1]), 0), cap))
    kv, cu, slots, positions, given = [], [0], np.full(T, -1, np.int64), np.zeros(T, np.int32), []
    end = taken = wanted = refused = 0
    for b, (a, n) in enumerate(zip(old, want)):
        a, n = min(max(int(a), 0), most * PAGE), max(int(n), 0)
        start, ok = end, n <= most * PAGE
        if ok and n > a:
            end += n - a
            ok = end <= T
            if ok and ring is not None and pages(n) > pages(a):
                wanted += pages(n) - pages(a)
                ok = wanted <= count
                if ok:
                    for i in range(pages(a), pages(n)):
                        table[b, i] = ring[(head + taken) % cap]
                        taken += 1
        if ok and ring is not None and n < a:
            given += [table[b, i] for i in range(pages(n), pages(a))]
        for t in range(min(start, T), min(end, T)):
            p = a + t - start
            positions[t] = p
            if ok and table[b, p // PAGE] >= 0:
                slots[t] = int(table[b, p // PAGE]) * PAGE + p % PAGE
        cu.append(min(end, T))
        kv.append(n if ok else a)
        refused += not ok
    if ring is None:
        return np.array(kv), np.array(cu), slots, positions, None
    for i, page in enumerate(given):
        ring[(head + count + i) % cap] = page
    return np.array(kv), np.array(cu), slots, positions, np.array([(head + taken) % cap, min(count - taken + len(given), cap), refused])


def phi(x):
    """Codes and scale bytes of x [..., d] (float64 values of bf16 numbers): nearest values of the formats, ties to the even code."""
    def nearest(v, values):
        lo = np.clip(np.searchsorted(values, v, side="right") - 1, 0, len(values) - 2)
        below, above = v - values[lo], values[lo + 1] - v
        return lo + ((above < below) | ((above == below) & (lo % 2 == 1)))
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    sc = nearest(np.abs(b).max(-1) / 6.0, E4M3[:127])
    s = E4M3[sc][..., None]
    code = nearest(np.where(s > 0, np.abs(b) / np.where(s > 0, s, 1.0), 0.0), GRID) + 8 * np.signbit(b)
    code = code.reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), sc.astype(np.uint8)


def value(codes, scales):
    c = np.stack([codes & 15, codes >> 4], axis=-1)
    return (E2M1[c].reshape(*scales.shape, 16) * E4M3[scales][..., None]).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def parts(cache, Hkv, d):
    """Codes [pages, heads, 2, 128, d/2] and scale bytes [pages, heads, 2, 128, d/16] of a cache (views)."""
    c = cache.reshape(-1, Hkv, 2, PAGE * (d // 2 + d // 16))
    n = PAGE * d // 2
    return c[..., :n].reshape(*c.shape[:-1], PAGE, d // 2), c[..., n:].reshape(*c.shape[:-1], PAGE, d // 16)


def random_cache(num_pages, Hkv, d, rng):
    """A cache of random codes and scales (2^-4 .. 2 times 1 .. 1.875): [pages, heads, 2, bytes of a part]."""
    c = rng.integers(0, 256, (num_pages, Hkv, 2, PAGE * (d // 2 + d // 16)), dtype=np.uint8)
    n = PAGE * d // 2
    c[..., n:] = rng.integers(24, 72, c[..., n:].shape, dtype=np.uint8)
    return c


def make_table(kv, rng, spare=2, extra_pages=1):
    """Pages of the sequences scattered over a cache; entries that are not needed point outside.  (table, number of pages)"""
    num_pages = sum(pages(n) for n in kv) + spare
    order = rng.permutation(num_pages).astype(np.int32)
    table = np.full((len(kv), max(max(pages(n) for n in kv), 1) + extra_pages), num_pages + 7, np.int32)
    table[::2][table[::2] > num_pages] = -3
    at = 0
    for b, n in enumerate(kv):
        table[b, :pages(n)] = order[at:at + pages(n)]
        at += pages(n)
    return table, num_pages


def bf16(x):
    """float64 array -> bf16 tensor on the CPU."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def gather(cache, table_row, n, Hkv, d):
    """K and V [n, Hkv, d] of one sequence, float64."""
    codes, scales = parts(cache, Hkv, d)
    pos = np.arange(n)
    pg, off = table_row[pos // PAGE], pos % PAGE
    live = (pg >= 0) & (pg < cache.shape[0])
    pg = np.where(live, pg, 0)
    return [np.where(live[:, None, None], value(codes[pg, :, i, off], scales[pg, :, i, off]), 0.0) for i in range(2)]


def attend(q, cu, cache, table, kv_lens, Hkv, causal, window, scale):
    """attnqat_fwd_kv4_ragged in 64 bits: (o, lse, weight) with weight = sum p |v|, which bounds the effect of rounding the probabilities.
    Rows that no sequence has: nan."""
    T, Hq, d = q.shape
    G = Hq // Hkv
    o, wt, lse = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full((T, Hq), np.nan)
    for b in range(len(kv_lens)):
        t0, n, kv = int(cu[b]), int(cu[b + 1] - cu[b]), int(kv_lens[b])
        if n == 0:
            continue
        if kv == 0:
            o[t0:t0 + n], wt[t0:t0 + n], lse[t0:t0 + n] = 0.0, 0.0, -np.inf
            continue
        k, v = gather(cache, table[b], kv, Hkv, d)
        at = kv - n + np.arange(n)[:, None]
        key = np.arange(kv)[None, :]
        see = np.ones((n, kv), bool)
        if causal:
            see &= key <= at
            if window:
                see &= key > at - window
        for hq in range(Hq):
            s = q[t0:t0 + n, hq] @ k[:, hq // G].T * scale
            s[~see] = -np.inf
            top = s.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0.0)
            p = np.exp(s - top)
            l = p.sum(1, keepdims=True)
            safe = np.where(l > 0, l, 1.0)
            o[t0:t0 + n, hq] = p @ v[:, hq // G] / safe
            wt[t0:t0 + n, hq] = p @ np.abs(v[:, hq // G]) / safe
            with np.errstate(divide="ignore"):
                lse[t0:t0 + n, hq] = (top + np.log(l))[:, 0]
    return o, lse, wt
