"""References of attention over chosen pages and of rotary positions (whole numbers and 64 bits, numpy)."""
import numpy as np

from tests import serve_util as S

PAGE = S.PAGE


def summary_parts(summary, Hkv, d):
    """Codes [pages, heads, d] and scales [pages, heads] of a summary (numpy uint8 -> int8, fp32)."""
    s = summary.reshape(-1, Hkv, d + 16)
    return s[..., :d].view(np.int8), np.ascontiguousarray(s[..., d:d + 4]).view(np.float32)[..., 0]


def mean_of_page(cache, page, Hkv, d):
    """Codes int8 [Hkv, d] and scales [Hkv] of a page, in whole numbers of 2^-10."""
    codes, scales = S.parts(cache, Hkv, d)
    v = S.value(codes[page, :, 0], scales[page, :, 0]) * 1024.0                              # [Hkv, 128, d]
    total = v.astype(np.int64)
    assert np.array_equal(total, v)
    total = total.sum(1)
    out, sc = np.zeros((Hkv, d), np.int8), np.zeros(Hkv, np.float32)
    for h in range(Hkv):
        big = int(np.abs(total[h]).max())
        e = big.bit_length() - 7
        for c in range(d):
            s = int(total[h, c])
            if e <= 0:
                code = s << -e
            else:
                code, rest, half = s >> e, s - (s >> e << e), 1 << (e - 1)
                code += rest > half or (rest == half and code & 1)
            out[h, c] = min(max(code, -127), 127)
        sc[h] = 2.0 ** (e - 17)
    return out, sc


def select(q, cu, codes, scale, table, kv_lens, Hkv, n_blocks, first, last, fill=-7):
    """attnqat_kv_select: blocks [T, Hkv, n_blocks] (rows of no sequence: fill).  Products of whole numbers; scores are exact in 64 bits."""
    T, Hq, d = q.shape
    G, num_pages = Hq // Hkv, codes.shape[0]
    out = np.full((T, Hkv, n_blocks), fill, np.int32)
    for b in range(len(kv_lens)):
        t0, n, kv = int(cu[b]), int(cu[b + 1] - cu[b]), int(kv_lens[b])
        for i in range(n):
            pos = kv - n + i
            for h in range(Hkv):
                row = out[t0 + i, h]
                row[:] = -1
                if pos < 0:
                    continue
                nb = pos // PAGE + 1
                if nb <= n_blocks:
                    row[:nb] = np.arange(nb)
                    continue
                x = q[t0 + i, h * G:(h + 1) * G]
                big = np.abs(x).max()
                q8 = np.clip(np.rint(x * 2.0 ** (6 - np.floor(np.log2(big)))) if big > 0 else x, -127, 127)
                ids = table[b, :nb]
                live = (ids >= 0) & (ids < num_pages)
                k = np.where(live[:, None], codes[np.where(live, ids, 0), h].astype(np.float64), 0.0)
                s = np.where(live, scale[np.where(live, ids, 0), h].astype(np.float64), 0.0) * (q8 @ k.T).max(0)
                rest = np.arange(first, nb - last)
                best = rest[np.argsort(-s[rest], kind="stable")[:n_blocks - first - last]]
                row[:] = np.sort(np.concatenate([np.arange(first), best, np.arange(nb - last, nb)]))
    return out


def attend(q, cu, cache, table, kv_lens, Hkv, blocks, scale, spread=False):
    """attnqat_fwd_kv4_sparse in 64 bits: (o, lse, weight) as serve_util.attend gives them.  spread: where scores spread widely, the weight counts the probabilities
    below 2^-25 of a row's largest too.  In fp16, with the largest at 2^11 or more, they are rounded by half a step of 2^-24, 2^-36 of the largest, which
    the sum that divides is at least: |error| <= 2^-36 sum |v|, 2^-25.5 sum |v| in terms of a weight that counts 2^-10.5."""
    T, Hq, d = q.shape
    G = Hq // Hkv
    o, wt, lse = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full((T, Hq), np.nan)
    for b in range(len(kv_lens)):
        t0, n, kv = int(cu[b]), int(cu[b + 1] - cu[b]), int(kv_lens[b])
        if n == 0:
            continue
        k, v = S.gather(cache, table[b], max(kv, 1), Hkv, d)
        for i in range(n):
            pos = kv - n + i
            for h in range(Hkv):
                blk = blocks[t0 + i, h].astype(np.int64)
                blk = np.unique(blk[(blk >= 0) & (blk * PAGE <= pos)]) if pos >= 0 else blk[:0]
                key = (blk[:, None] * PAGE + np.arange(PAGE)).reshape(-1)
                key = key[key <= pos]
                hq = slice(h * G, (h + 1) * G)
                if key.size == 0:
                    o[t0 + i, hq], wt[t0 + i, hq], lse[t0 + i, hq] = 0.0, 0.0, -np.inf
                    continue
                s = q[t0 + i, hq] @ k[key, h].T * scale
                top = s.max(1, keepdims=True)
                p = np.exp(s - top)
                l = p.sum(1, keepdims=True)
                o[t0 + i, hq], wt[t0 + i, hq], lse[t0 + i, hq] = p @ v[key, h] / l, p @ np.abs(v[key, h]) / l, (top + np.log(l))[:, 0]
                if spread:
                    wt[t0 + i, hq] += 2.0 ** -25.5 * np.abs(v[key, h]).sum(0)
    return o, lse, wt


def turned(x, positions, freqs, axis, layout, sign=1.0):
    """x [L, heads, d] turned (64 bits), and |a| + |b| of every value's pair, which bounds what sine, cosine and products may be off."""
    y, size = x.copy(), np.zeros_like(x)
    n = len(freqs)
    for i, (f, a) in enumerate(zip(freqs, axis)):
        u, w = (2 * i, 2 * i + 1) if layout == "paired" else (i, i + n)
        # the angle modulo a turn in more than 64 bits: p f may be millions of radians
        t = np.array([float(np.longdouble(int(p)) * np.longdouble(f) % (2 * np.longdouble("3.14159265358979323846264338327950288"))) for p in positions[:, a]])[:, None]
        c, s = np.cos(t), sign * np.sin(t)
        y[..., u], y[..., w] = x[..., u] * c - x[..., w] * s, x[..., u] * s + x[..., w] * c
        size[..., u] = size[..., w] = np.abs(x[..., u]) + np.abs(x[..., w])
    return y, size
