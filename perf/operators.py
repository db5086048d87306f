"""Serving steps over the NVFP4 KV cache whose sequences bring different numbers of new positions: what is timed, and the
operators in elementary torch operations.

Kinds of case (``op``)
  plan    page table, slot map and positions of a step from the lengths of its requests; pages are taken from and given back to
          a ring of free pages
  append  K and V of the step's tokens, quantized into their slots; what the slots then hold is read back
  read    every position of some sequences, out of the cache as bf16
  attn    attention of the step's queries over the cache; Q and the probabilities are not quantized

A page holds 128 positions of one sequence for all kv heads: per head K codes [128][d/2], K scale bytes [128][d/16], V codes,
V scale bytes (E2M1 elements, one E4M3 scale per 16 of them).
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 128
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)        # the magnitudes of E2M1


def listed():
    plan = lambda name, mix, B, q, kv, shrink=0.0, decode=0.0, pool=1.0: {  # noqa: E731
        "name": name, "op": "plan", "mix": mix, "B": B, "q_min": q[0], "q_max": q[1], "kv_min": kv[0], "kv_max": kv[1],
        "shrink": shrink, "decode": decode, "pool": pool}
    rows = lambda name, op, mix, B, Hkv, d, q, kv, pad=0, fused=True, decode=0.0: {  # noqa: E731
        "name": name, "op": op, "mix": mix, "B": B, "Hkv": Hkv, "d": d, "q_min": q[0], "q_max": q[1], "kv_min": kv[0], "kv_max": kv[1],
        "pad": pad, "fused": fused, "decode": decode}
    attn = lambda name, mix, B, Hq, Hkv, d, q, kv, decode=0.0, causal=True, window=0, fused=True, dist="normal": {  # noqa: E731
        "name": name, "op": "attn", "mix": mix, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "q_min": q[0], "q_max": q[1], "kv_min": kv[0],
        "kv_max": kv[1], "decode": decode, "causal": causal, "window": window, "fused": fused, "dist": dist}
    return [
        # every step of a small server: 24 requests grow by one token
        plan("plan_decode", 1, 24, (1, 1), (60, 5000)),
        # a step of a large one: 700 requests, prompts cut into chunks among decodes, drafted tokens taken back, pages running short
        plan("plan_mixed", 2, 700, (1, 2000), (1, 16000), shrink=0.2, decode=0.6, pool=0.7),
        # the tokens of a decode step of 32 sequences (the grouped-query language model), padded to the size a graph was captured for
        rows("append_decode", "append", 3, 32, 8, 128, (1, 1), (4096, 16384), pad=8),
        # prompts of nine requests at once, K and V views of one projection
        rows("append_prompts", "append", 4, 9, 8, 128, (150, 6000), (150, 6000)),
        # one short conversation leaves for a kernel that takes bf16
        rows("read_short", "read", 5, 1, 8, 128, (1, 1), (777, 777), fused=False),
        # long contexts moved out of the cache
        rows("read_contexts", "read", 6, 5, 8, 128, (1, 1), (9000, 40000), fused=False),
        # one user with a conversation of about 3000 tokens, one new token: latency
        attn("attn_single", 7, 1, 32, 8, 128, (1, 1), (3000, 3000)),
        # a decode step of 32 sequences of 4k - 16k keys
        attn("attn_decode32", 8, 32, 32, 8, 128, (1, 1), (4096, 16384), dist="k_outliers"),
        # drafted tokens to be checked: one to six queries a sequence, heads of 64
        attn("attn_drafts", 9, 40, 16, 4, 64, (1, 6), (300, 9000)),
        # chunked prefill beside decodes: most sequences bring one token, some a piece of a prompt
        attn("attn_mixed", 10, 28, 32, 8, 128, (100, 1500), (1500, 16000), decode=0.85),
        # whole prompts of odd lengths, nothing in the cache before them
        attn("attn_prompts", 11, 6, 32, 8, 128, (700, 6000), (700, 6000), dist="k_outliers"),
        # a layer with a sliding window over long conversations, decodes and short chunks, one kv head per four query heads of 64
        attn("attn_window", 12, 24, 16, 4, 64, (1, 300), (2000, 50000), decode=0.5, window=1024, fused=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same kinds: sizes spread over the logarithm of their range, none dearer than the largest listed case of
    its kind."""
    op = rng.choice(["plan", "append", "read", "attn", "attn", "attn", "attn"])
    mix = rng.randrange(1 << 30)
    d = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 12])
    if op == "plan":
        q = sorted((1, _log_int(rng, 1, 2000)))
        kv = sorted(_log_int(rng, 1, 16000) for _ in range(2))
        return {"op": op, "mix": mix, "B": _log_int(rng, 1, 700), "q_min": q[0], "q_max": q[1], "kv_min": kv[0], "kv_max": kv[1],
                "shrink": rng.choice([0.0, 0.3]), "decode": rng.choice([0.0, 0.5, 0.9]), "pool": rng.choice([1.0, 1.0, 0.5])}
    if op in ("append", "read"):
        top = 20000 * 8 // Hkv if op == "append" else 100000 * 8 // Hkv
        B = _log_int(rng, 1, 64)
        a, b = sorted(_log_int(rng, 1, max(2, min(40000, top // B))) for _ in range(2))
        return {"op": op, "mix": mix, "B": B, "Hkv": Hkv, "d": d, "q_min": a if op == "append" else 1, "q_max": b if op == "append" else 1,
                "kv_min": a, "kv_max": b + 500 if op == "append" else b, "pad": rng.choice([0, 5]), "fused": rng.random() < 0.5,
                "decode": rng.choice([0.0, 0.7]) if op == "append" else 0.0}
    G = rng.choice([1, 1, 2, 4, 4, 8, 16])
    while G * Hkv > 64:
        G //= 2
    B = _log_int(rng, 1, 64)
    top = max(700, min(50000, int(32 * 10000 * 8 * 128 / (B * Hkv * d))))
    kv = sorted(_log_int(rng, 200, top) for _ in range(2))
    kind = rng.choice(["decode", "decode", "draft", "mixed", "prompt"])
    c = {"op": op, "mix": mix, "B": B, "Hq": G * Hkv, "Hkv": Hkv, "d": d, "q_min": 1, "q_max": 1, "kv_min": kv[0], "kv_max": kv[1],
         "decode": 0.0, "causal": rng.random() < 0.85, "window": 0, "fused": rng.random() < 0.5,
         "dist": rng.choice(["normal", "k_outliers", "t3"])}
    if kind == "draft":
        c["q_max"] = rng.choice([2, 4, 8])
    elif kind == "mixed":
        c["q_max"], c["decode"] = _log_int(rng, 16, 1500), 0.8
    elif kind == "prompt":
        c["q_min"], c["q_max"] = 16, _log_int(rng, 16, 4000)
    if kind in ("mixed", "prompt"):                              # no more pairs than attn_mixed has
        c["B"] = min(B, 16)
        c["kv_min"], c["kv_max"] = min(c["kv_min"], 12000), min(c["kv_max"], 16000)
        while _pairs(c) * G * Hkv * d > 5.5e10:
            if c["B"] > 1:
                c["B"] //= 2
            else:
                c["q_max"] = max(16, c["q_max"] // 2)
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log_int(rng, 64, 4096)
    return c


def _lens(c):
    """(new positions, positions in all) of every sequence of a case."""
    rng = random.Random(c["mix"])
    out = []
    for _ in range(c["B"]):
        kv = _log_int(rng, c["kv_min"], c["kv_max"])
        n = 1 if rng.random() < c["decode"] else _log_int(rng, c["q_min"], c["q_max"])
        if c["op"] == "append" and c["q_max"] > 1:
            kv = max(kv, n)
        out.append((min(n, kv), kv))
    if c["op"] in ("append", "attn") and c["kv_min"] == c["q_min"] and c["kv_max"] == c["q_max"]:      # whole prompts
        out = [(kv, kv) for _, kv in out]
    return out


def _pairs(c):
    """Visible (query, key) pairs of an attention case, for one head."""
    total = 0
    for n, kv in _lens(c):
        if not c["causal"]:
            total += n * kv
        else:
            w = c["window"]
            total += sum(min(kv - n + i + 1, w) if w else kv - n + i + 1 for i in range(n))
    return total


def _pages(n):
    return (n + PAGE - 1) // PAGE


def work(case):
    c = case
    if c["op"] == "plan":
        tokens = sum(n for n, _ in _lens(c))
        moved = sum(_pages(kv) - _pages(kv - n) for n, kv in _lens(c))
        return {"bytes": 16 * c["B"] + 12 * tokens + 8 * moved, "flops": 0}
    packed = c["Hkv"] * (c["d"] // 2 + c["d"] // 16)
    if c["op"] == "append":
        tokens = sum(n for n, _ in _lens(c)) + c["pad"]          # in as bf16, packed; read back: packed in, bf16 out
        return {"bytes": 2 * tokens * (2 * 2 * c["Hkv"] * c["d"] + 2 * packed + 8), "flops": 0}
    if c["op"] == "read":
        tokens = sum(kv for _, kv in _lens(c)) + c["pad"]
        return {"bytes": tokens * (2 * 2 * c["Hkv"] * c["d"] + 2 * packed + 8), "flops": 0}
    seen = sum(min(kv, n + c["window"] - 1) if c["window"] else kv for n, kv in _lens(c))
    tokens = sum(n for n, _ in _lens(c))
    return {"bytes": 2 * seen * packed + tokens * c["Hq"] * (4 * c["d"] + 4), "flops": 4 * c["d"] * c["Hq"] * _pairs(c)}


# ---------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _values(shape, dist, what, g):
    """bf16 [tokens, heads, d].  normal: N(0,1).  k_outliers: four channels of K x20.  t3: 0.5 Student-t with 3 degrees of freedom."""
    x = torch.randn(shape, generator=g, device=DEV)
    if dist == "k_outliers" and what == "k":
        x[..., torch.randperm(shape[-1], generator=g, device=DEV)[:4]] *= 20.0
    elif dist == "t3":
        z = sum(torch.randn(shape, generator=g, device=DEV).square_() for _ in range(3))
        x = 0.5 * x / (z / 3.0).sqrt()
    return x.to(torch.bfloat16)


def _split(T, heads, d, g, dist, fused):
    """q-or-nothing, k, v [T, heads, d] as a projection leaves them: views of one tensor (fused) or tensors of their own."""
    parts = [_values((T, h, d), dist, w, g) for w, h in zip("qkv", heads)]
    if not fused:
        return parts
    return list(torch.cat(parts, dim=1).split(list(heads), dim=1))


def _tables(lens, g):
    """A cache with room for the sequences, their pages scattered over it: page table [B, max_pages], number of pages."""
    max_pages = max(_pages(kv) for kv in lens) + 1
    num_pages = sum(_pages(kv) for kv in lens) + 3
    order = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, kv in enumerate(lens):
        table[b, :_pages(kv)] = order[at:at + _pages(kv)]
        at += _pages(kv)
    return table, num_pages


def _parts(cache, Hkv, d):
    """Views of a cache's codes [pages, heads, 2, 128, d/2] and scale bytes [pages, heads, 2, 128, d/16]."""
    c = cache.view(-1, Hkv, 2, PAGE * (d // 2 + d // 16))
    n = PAGE * d // 2
    return c[..., :n].unflatten(-1, (PAGE, d // 2)), c[..., n:].unflatten(-1, (PAGE, d // 16))


def _cache(num_pages, Hkv, d, g, dist="normal"):
    """A cache full of quantized K and V."""
    cache = torch.empty(num_pages * Hkv * 2 * PAGE * (d // 2 + d // 16), dtype=torch.uint8, device=DEV)
    codes, scales = _parts(cache, Hkv, d)
    step = max(1, (1 << 26) // (Hkv * PAGE * d))
    for p in range(0, num_pages, step):
        n = min(step, num_pages - p)
        for i, what in enumerate("kv"):
            codes[p:p + n, :, i], scales[p:p + n, :, i] = _pack(_values((n, Hkv, PAGE, d), dist, what, g))
    return cache


def _slots_of(table, spans):
    """Slots of positions [a, b) of every sequence, one after another."""
    out = []
    for i, (a, b) in enumerate(spans):
        p = torch.arange(a, b, device=DEV)
        out.append(table[i, p // PAGE].long() * PAGE + p % PAGE)
    return torch.cat(out)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prefix(x):
    out = [0]
    for n in x:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    c, g, lens = case, _generator(seed), _lens(case)
    if c["op"] == "plan":
        return _prepare_plan(c, lens, g, seed)
    Hkv, d, B = c["Hkv"], c["d"], c["B"]
    s = {"case": c, "Hkv": Hkv, "d": d}
    if c["op"] in ("append", "read"):
        table, s["num_pages"] = _tables([kv for _, kv in lens], g)
        s["cache"] = _cache(s["num_pages"], Hkv, d, g)
        s["slots"] = _slots_of(table, [(kv - n, kv) if c["op"] == "append" else (0, kv) for n, kv in lens])
        if c["pad"]:
            s["slots"] = torch.cat([s["slots"], torch.full((c["pad"],), -1, dtype=torch.int64, device=DEV)])
        T = s["slots"].numel()
        if c["op"] == "append":
            _, s["k"], s["v"] = _split(T, (2 * Hkv, Hkv, Hkv), d, g, "normal", c["fused"])
        s["out"] = tuple(torch.empty((T, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return s
    n, kv = [a for a, _ in lens], [b for _, b in lens]
    s["n"], s["kv"] = n, kv                                       # (the plain form walks over the sequences)
    s["table"], s["num_pages"] = _tables(kv, g)
    s["cache"] = _cache(s["num_pages"], Hkv, d, g, c["dist"])
    T = sum(n)
    s["q"] = _split(T, (c["Hq"], Hkv, Hkv), d, g, c["dist"], c["fused"])[0] if c["fused"] else _values((T, c["Hq"], d), c["dist"], "q", g)
    s["cu_q"], s["kv_lens"], s["max_q"] = _ints(_prefix(n)), _ints(kv), max(n)
    s["scale"] = 1.0 / math.sqrt(d)
    s["out"] = (torch.empty((T, c["Hq"], d), dtype=torch.bfloat16, device=DEV), torch.empty((T, c["Hq"]), dtype=torch.float32, device=DEV))
    if own:
        import paper_2603_00040_amd as aq
        s["workspace"] = torch.empty(aq.kv4_ragged_workspace_bytes(T, B, c["Hq"], Hkv, s["max_q"], s["table"].shape[1], d),
                                     dtype=torch.uint8, device=DEV)
    return s


def _prepare_plan(c, lens, g, seed):
    rng = random.Random(seed)
    old, new = [], []
    for n, kv in lens:
        if rng.random() < c["shrink"]:
            old.append(kv)
            new.append(max(0, kv - n))
        else:
            old.append(kv - n)
            new.append(kv)
    max_pages = max(_pages(kv) for _, kv in lens) + 1
    held = sum(_pages(o) for o in old)
    need = sum(max(0, _pages(b) - _pages(a)) for a, b in zip(old, new))
    free = max(1, int(c["pool"] * need) + 1)
    num_pages = held + max(free, need) + 2
    order = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((c["B"], max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, o in enumerate(old):
        table[b, :_pages(o)] = order[at:at + _pages(o)]
        at += _pages(o)
    head = rng.randrange(num_pages)
    ring = torch.full((num_pages,), -1, dtype=torch.int32, device=DEV)
    where = (head + torch.arange(free, device=DEV)) % num_pages
    ring[where] = order[at:at + free]
    T = sum(n for n, _ in lens)
    s = {"case": c, "kv_lens": _ints(old), "new_lens": _ints(new), "table": table, "ring": ring, "ring_state": _ints([head, free, 0]), "T": T}
    e = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
    s["out"] = (e(c["B"]), e(c["B"] + 1), e(T, torch.int64), e(T), e(3))
    if own:
        import paper_2603_00040_amd as aq
        s["workspace"] = e(aq.page_plan_workspace_bytes(c["B"]), torch.uint8)
    return s


# ---------------------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2603_00040_amd as aq
        s = state
        if op == "plan":
            kv, cu, slots, positions, ring_state = aq.attnqat_page_plan(s["kv_lens"], s["new_lens"], s["table"], s["T"], free=(s["ring"], s["ring_state"]),
                                                                        workspace=s["workspace"], out=s["out"])
            return {"kv_lens": kv, "cu": cu, "slots": slots, "positions": positions, "ring_state": ring_state, "table": s["table"], "ring": s["ring"]}
        if op in ("append", "read"):
            if op == "append":
                aq.attnqat_kv_cache_append(s["k"], s["v"], s["cache"], s["slots"], num_pages=s["num_pages"])
            k, v = aq.attnqat_kv_cache_read(s["cache"], s["slots"], s["Hkv"], s["d"], num_pages=s["num_pages"], out=s["out"])
            return {"k": k, "v": v}
        o, lse = aq.attnqat_fwd_kv4_ragged(s["q"], s["cu_q"], s["cache"], s["num_pages"], s["table"], s["kv_lens"], s["Hkv"], s["case"]["causal"],
                                           max_q=s["max_q"], window=s["case"]["window"], scale=s["scale"], workspace=s["workspace"], out=s["out"])
        return {"o": o, "lse": lse}
    if op == "plan":
        return _plan(state)
    if op == "append":
        _append(state)
    if op in ("append", "read"):
        return _read(state)
    return _attend(state)


# The plain forms.
def _pack(x):
    """phi of x [..., d] bf16: codes and scale bytes.  (Quotients of a bf16 number by 6 or by an E4M3 scale are no nearer than 2^-13 to a
    boundary that they are not on: 32 bits decide as real numbers would.)"""
    b = x.float().unflatten(-1, (-1, 16))
    scale = (b.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    r = b.abs() / scale.float().clamp(min=2.0 ** -9)[..., None]
    r = torch.where(scale.float()[..., None] > 0, r, 0.0)
    code = ((r > 0.25).byte() + (r >= 0.75).byte() + (r > 1.25).byte() + (r >= 1.75).byte() + (r > 2.5).byte() + (r >= 3.5).byte() + (r > 5.0).byte()
            + 8 * torch.signbit(b).byte()).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.view(torch.uint8)


def _unpack(codes, scales):
    lut = torch.tensor(GRID + tuple(-x for x in GRID), device=DEV)
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    return (lut[c].unflatten(-1, (-1, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _places(s):
    inside = (s["slots"] >= 0) & (s["slots"] < s["num_pages"] * PAGE)
    slot = torch.where(inside, s["slots"], 0)
    return inside, slot // PAGE, slot % PAGE


def _append(s):
    inside, page, off = _places(s)
    codes, scales = _parts(s["cache"], s["Hkv"], s["d"])
    if s["case"]["pad"]:                                          # (the padding rows lie at the end)
        n = inside.numel() - s["case"]["pad"]
        page, off = page[:n], off[:n]
    n = page.numel()
    for i, x in enumerate((s["k"], s["v"])):
        c, sc = _pack(x[:n])
        codes[page, :, i, off] = c
        scales[page, :, i, off] = sc


def _read(s):
    inside, page, off = _places(s)
    codes, scales = _parts(s["cache"], s["Hkv"], s["d"])
    out = []
    for i in range(2):
        y = _unpack(codes[page, :, i, off], scales[page, :, i, off])
        out.append(torch.where(inside[:, None, None], y, 0.0).to(torch.bfloat16))
    return {"k": out[0], "v": out[1]}


def _plan(s):
    table, ring, st, T = s["table"], s["ring"], s["ring_state"].long(), s["T"]
    B, most = table.shape
    cap = ring.numel()
    old, new = s["kv_lens"].long().clamp(0, most * PAGE), s["new_lens"].long().clamp(min=0)
    bad = new > most * PAGE
    grow = torch.where(bad, 0, (new - old).clamp(min=0))
    end = grow.cumsum(0)
    late = (grow > 0) & (end > T)
    p_old, p_new = (old + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    need = torch.where(bad | late, 0, (p_new - p_old).clamp(min=0))
    upto = need.cumsum(0)
    ok = ~(bad | late | ((need > 0) & (upto > st[1])))
    back = (p_old - p_new).clamp(min=0)
    j = torch.arange(most, device=DEV)
    give = (j >= p_new[:, None]) & (j < p_old[:, None])           # pages given back: behind the free ones
    where = (st[0] + st[1] + (back.cumsum(0) - back - p_new)[:, None] + j) % cap
    wider = torch.cat([ring, ring.new_zeros(1)])
    wider.scatter_(0, torch.where(give, where, cap).flatten(), table.flatten())
    take = ok[:, None] & (j >= p_old[:, None]) & (j < p_new[:, None])
    where = (st[0] + (upto - need - p_old)[:, None] + j) % cap
    table.copy_(torch.where(take, ring[where], table))
    ring.copy_(wider[:cap])
    taken = torch.where(ok, need, 0).sum()
    state = torch.stack([(st[0] + taken) % cap, st[1] - taken + back.sum(), (~ok).sum()]).int()
    cu = torch.cat([end.new_zeros(1), end.clamp(max=T)])
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=B - 1)
    live = t < cu[B]
    pos = torch.where(live, old[b] + t - cu[b], 0)
    page = table[b, (pos // PAGE).clamp(max=most - 1)].long()
    slots = torch.where(live & ok[b] & (page >= 0), page * PAGE + pos % PAGE, -1)
    return {"kv_lens": torch.where(ok, new, old).int(), "cu": cu.int(), "slots": slots, "positions": pos.int(), "ring_state": state, "table": table, "ring": ring}


def _attend(s):
    c, Hkv, d = s["case"], s["Hkv"], s["d"]
    G = c["Hq"] // Hkv
    o, lse = s["out"]
    codes, scales = _parts(s["cache"], Hkv, d)
    at = 0
    for b, (n, kv) in enumerate(zip(s["n"], s["kv"])):
        first = max(0, kv - n + 1 - c["window"]) // PAGE if c["window"] else 0      # pages in front of every window
        ids = s["table"][b, first:_pages(kv)].long()
        k, v = (_unpack(codes[ids, :, i], scales[ids, :, i]).transpose(0, 1).flatten(1, 2) for i in range(2))
        key = torch.arange(first * PAGE, _pages(kv) * PAGE, device=DEV)
        rows = max(1, (1 << 28) // (c["Hq"] * key.numel()))
        for r in range(0, n, rows):
            m = min(rows, n - r)
            q = s["q"][at + r:at + r + m].float().unflatten(1, (Hkv, G)).permute(1, 0, 2, 3).flatten(1, 2)       # [Hkv, m G, d]
            x = torch.matmul(q, k.transpose(1, 2)).mul_(s["scale"])
            here = kv - n + r + torch.arange(m, device=DEV).repeat_interleave(G)[:, None]
            hidden = key >= kv
            if c["causal"]:
                hidden = hidden | (key > here)
                if c["window"]:
                    hidden = hidden | (key <= here - c["window"])
            x.masked_fill_(hidden, -math.inf)
            top = x.amax(-1, keepdim=True)
            p = x.sub_(top).exp_()
            l = p.sum(-1, keepdim=True)
            y = torch.matmul(p, v) / l
            o[at + r:at + r + m] = y.unflatten(1, (m, G)).permute(1, 0, 2, 3).flatten(1, 2).to(torch.bfloat16)
            lse[at + r:at + r + m] = (top + l.log()).unflatten(1, (m, G)).permute(1, 0, 2, 3).flatten(1)
        at += n
    return {"o": o, "lse": lse}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "plan":
        return _exact_plan(s)
    if c["op"] == "append":
        pages = s["slots"] >= 0
        return {n: torch.where(pages[:, None, None], _exact_phi(s[n]), 0.0) for n in "kv"}
    Hkv, d = c["Hkv"], c["d"]
    # every byte's value by its definition: sign, exponent, mantissa
    e4m3 = torch.tensor([math.nan if i & 127 == 127 else (-1) ** (i >> 7) * ((i & 7) * 2.0 ** -9 if (i >> 3) & 15 == 0
                         else (8 + (i & 7)) * 2.0 ** (((i >> 3) & 15) - 10)) for i in range(256)], dtype=torch.float64, device=DEV)
    e2m1 = torch.tensor([(-1) ** (i >> 3) * ((i & 1) * 0.5 if (i >> 1) & 3 == 0 else (2 + (i & 1)) * 2.0 ** (((i >> 1) & 3) - 2)) for i in range(16)],
                        dtype=torch.float64, device=DEV)
    half = Hkv * 2 * PAGE * (d // 2 + d // 16)
    cache = s["cache"].view(s["num_pages"], half)

    def rows(page, off, which):                                   # [tokens, Hkv, d]
        base = (torch.arange(Hkv, device=DEV) * 2 + which) * PAGE * (d // 2 + d // 16)
        at = base[None, :, None] + off[:, None, None] * (d // 2) + torch.arange(d, device=DEV) // 2
        byte = cache[page[:, None, None], at].long()
        nib = torch.where(torch.arange(d, device=DEV) % 2 == 0, byte % 16, byte // 16)
        sc = cache[page[:, None, None], base[None, :, None] + PAGE * (d // 2) + off[:, None, None] * (d // 16) + torch.arange(d, device=DEV) // 16].long()
        return e2m1[nib] * e4m3[sc]

    if c["op"] == "read":
        if s["slots"].numel() * Hkv * d > 1 << 28:
            return None
        live = s["slots"] >= 0
        at = s["slots"].clamp(min=0)
        return {n: torch.where(live[:, None, None], rows(at // PAGE, at % PAGE, i), 0.0) for i, n in enumerate("kv")}
    if _pairs(c) * c["Hq"] * d > 1.0e12:
        return None
    G = c["Hq"] // Hkv
    o = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    first_row = 0
    for b, (n, kv) in enumerate(zip(s["n"], s["kv"])):
        pos = torch.arange(kv, device=DEV)
        page, off = s["table"][b].long()[pos // PAGE], pos % PAGE
        k, v = rows(page, off, 0), rows(page, off, 1)
        for h in range(Hkv):
            kh, vh = k[:, h].contiguous(), v[:, h].contiguous()
            for g in range(G):
                q = s["q"][first_row:first_row + n, h * G + g].double()
                x = (q @ kh.t()) * s["scale"]
                if c["causal"]:
                    gap = (kv - n + torch.arange(n, device=DEV))[:, None] - pos[None, :]      # how far behind the query a key lies
                    x[(gap < 0) | ((gap >= c["window"]) if c["window"] else (gap < 0))] = -math.inf
                z = torch.logsumexp(x, dim=1)
                o[first_row:first_row + n, h * G + g] = torch.exp(x - z[:, None]) @ vh
                lse[first_row:first_row + n, h * G + g] = z
        first_row += n
    return {"o": o, "lse": lse}


def _exact_phi(x):
    """phi^-1(phi(x)) with both roundings decided among all values of the formats."""
    scales = torch.tensor([i * 2.0 ** -9 for i in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
                          dtype=torch.float64, device=DEV)
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)

    def nearest(v, values):                                       # ties to the even index
        lo = (torch.searchsorted(values, v.contiguous(), right=True) - 1).clamp(0, values.numel() - 2)
        below, above = v - values[lo], values[lo + 1] - v
        up = (above < below) | ((above == below) & (lo % 2 == 1))
        return values[lo + up.long()]

    b = x.double().unflatten(-1, (-1, 16))
    s = nearest(b.abs().amax(-1, keepdim=True) / 6.0, scales)
    r = torch.where(s > 0, b.abs() / torch.where(s > 0, s, 1.0), 0.0)
    return (torch.sign(b) * nearest(r, grid) * s).flatten(-2)


def _exact_plan(s):
    """The same step, request after request."""
    old, want, table, ring = s["kv_lens"].tolist(), s["new_lens"].tolist(), s["table"].tolist(), s["ring"].tolist()
    head, count, _ = s["ring_state"].tolist()
    most, cap, T = len(table[0]), len(ring), s["T"]
    kv, cu, slots, positions, given, refused, taken, wanted, end = [], [0], [-1] * T, [0] * T, [], 0, 0, 0, 0
    for b, (a, n) in enumerate(zip(old, want)):
        pa, pn = _pages(a), _pages(n)
        fine = n <= most * PAGE
        start = end
        if fine and n > a:
            end += n - a
            fine = end <= T
            if fine and pn > pa:
                wanted += pn - pa
                fine = wanted <= count
                if fine:
                    for i in range(pa, pn):
                        table[b][i] = ring[(head + taken) % cap]
                        taken += 1
        given += table[b][pn:pa]
        for t in range(min(start, T), min(end, T)):
            p = a + t - start
            positions[t] = p
            if fine and table[b][p // PAGE] >= 0:
                slots[t] = table[b][p // PAGE] * PAGE + p % PAGE
        cu.append(min(end, T))
        kv.append(n if fine else a)
        refused += not fine
    for i, page in enumerate(given):
        ring[(head + count + i) % cap] = page
    state = [(head + taken) % cap, count - taken + len(given), refused]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"kv_lens": i32(kv), "cu": i32(cu), "slots": torch.tensor(slots, dtype=torch.int64, device=DEV), "positions": i32(positions),
            "ring_state": i32(state), "table": i32(table), "ring": i32(ring)}
