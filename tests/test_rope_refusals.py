"""What the entry points of rotary positions refuse, by status and before anything is enqueued (no GPU is touched: the pointers are numbers)."""
import ctypes
import math
from fractions import Fraction

import pytest

import paper_2603_00040_amd as aq

P = 1 << 24
PI2 = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")


def _rope(pairs=32, axes=1, layout=0):
    return aq.Rope(pairs, axes, layout, 0, (ctypes.c_uint64 * 64)(*[1 << 60] * 64))


def _call(back=False, **kw):
    # [B,L,heads,d] buffers: q of 4 heads, k of 2, V of 2 in one; contiguous results
    a = dict(q=P, qs=(8192, 64, 512), k=P + 512, ks=(8192, 64, 512), B=2, Hq=4, Hkv=2, L=16, d=64, dtype=0, pos=2 * P, pos_batch=0, rope=_rope(),
             qo=3 * P, qos=(4096, 1024, 64), ko=4 * P, kos=(2048, 1024, 64))
    a.update(kw)
    rope = None if a["rope"] is None else ctypes.addressof(a["rope"])
    f = aq.lib().attnqat_rope_bwd if back else aq.lib().attnqat_rope_fwd
    return f(a["q"], *a["qs"], a["k"], *a["ks"], a["B"], a["Hq"], a["Hkv"], a["L"], a["d"], a["dtype"], a["pos"], a["pos_batch"], rope, a["qo"], *a["qos"], a["ko"], *a["kos"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), aq.EINVAL), (dict(k=None), aq.EINVAL), (dict(pos=None), aq.EINVAL), (dict(rope=None), aq.EINVAL), (dict(qo=None), aq.EINVAL), (dict(ko=None), aq.EINVAL),
    (dict(B=0), aq.EINVAL), (dict(L=-1), aq.EINVAL), (dict(Hq=0), aq.EINVAL), (dict(Hkv=-1), aq.EINVAL), (dict(d=96), aq.ESHAPE), (dict(dtype=1), aq.EDTYPE),
    (dict(B=1 << 14, L=(1 << 14) + 1), aq.ESHAPE), (dict(Hq=65536), aq.ESHAPE), (dict(q=P + 8), aq.EINVAL), (dict(qo=3 * P + 2), aq.EINVAL), (dict(pos=2 * P + 2), aq.EINVAL),
    (dict(pos_batch=-1), aq.EINVAL), (dict(qs=(8192, 60, 512)), aq.EINVAL), (dict(qs=(-8192, 64, 512)), aq.EINVAL), (dict(qs=(1 << 60, 64, 512)), aq.EINVAL),
    (dict(qos=(4096, 1024, 32)), aq.EINVAL), (dict(qos=(4096, 512, 64)), aq.EINVAL), (dict(qos=(0, 1024, 64)), aq.EINVAL), (dict(qos=(4096, 1024, 0)), aq.EINVAL),
    (dict(rope=_rope(pairs=0)), aq.EINVAL), (dict(rope=_rope(pairs=33)), aq.EINVAL), (dict(rope=_rope(axes=0)), aq.EINVAL), (dict(rope=_rope(axes=5)), aq.EINVAL),
    (dict(rope=_rope(layout=2)), aq.EINVAL),
    (dict(rope=_rope(pairs=12, layout=1)), aq.ESHAPE),
    # outputs over inputs, positions and each other
    (dict(qo=P), aq.EINVAL), (dict(qo=P + 512, qos=(8192, 64, 512)), aq.EINVAL), (dict(qo=P + 128, qos=(8192, 64, 512)), aq.EINVAL), (dict(ko=P, kos=(8192, 64, 512)), aq.EINVAL),
    (dict(ko=3 * P + 4096), aq.EINVAL), (dict(qo=2 * P), aq.EINVAL), (dict(qo=P, qos=(8192, 512, 64)), aq.EINVAL),
    (dict(qo=3 * P, qos=(8192, 64, 512), ko=3 * P + 384, kos=(8192, 64, 512)), aq.EINVAL)])
@pytest.mark.parametrize("back", [False, True])
def test_rope(kw, code, back):
    assert _call(back, **kw) == code


def test_no_tokens_no_work():
    assert _call(L=0) == aq.OK and _call(L=0, q=None, qo=None, pos=None) == aq.OK


def _append(**kw):
    a = dict(q=P, qt=512, qh=64, k=P + 512, kt=512, kh=64, v=P + 768, vt=512, vh=64, T=6, Hq=4, Hkv=2, d=64, dtype=0, pos=2 * P, rope=_rope(), cache=3 * P, pages=4, slots=4 * P,
             qo=5 * P, qot=256, qoh=64)
    a.update(kw)
    rope = None if a["rope"] is None else ctypes.addressof(a["rope"])
    return aq.lib().attnqat_kv_cache_append_rope(a["q"], a["qt"], a["qh"], a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], a["T"], a["Hq"], a["Hkv"], a["d"], a["dtype"], a["pos"], rope,
                                                 a["cache"], a["pages"], a["slots"], a["qo"], a["qot"], a["qoh"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), aq.EINVAL), (dict(k=None), aq.EINVAL), (dict(v=None), aq.EINVAL), (dict(qo=None), aq.EINVAL), (dict(pos=None), aq.EINVAL), (dict(rope=None), aq.EINVAL),
    (dict(cache=None), aq.EINVAL), (dict(slots=None), aq.EINVAL), (dict(T=-1), aq.EINVAL), (dict(Hq=-1), aq.EINVAL), (dict(Hkv=0), aq.EINVAL), (dict(pages=0), aq.EINVAL),
    (dict(dtype=3), aq.EDTYPE), (dict(d=32), aq.ESHAPE), (dict(T=1 << 28), aq.ESHAPE), (dict(Hq=1 << 17), aq.ESHAPE), (dict(Hkv=1 << 17), aq.ESHAPE),
    (dict(q=P + 4), aq.EINVAL), (dict(qo=5 * P + 8), aq.EINVAL), (dict(cache=3 * P + 4), aq.EINVAL), (dict(slots=4 * P + 4), aq.EINVAL), (dict(pos=2 * P + 1), aq.EINVAL),
    (dict(qt=500), aq.EINVAL), (dict(qot=128), aq.EINVAL), (dict(qoh=32), aq.EINVAL), (dict(rope=_rope(pairs=40)), aq.EINVAL), (dict(rope=_rope(pairs=20, layout=1)), aq.ESHAPE),
    (dict(qo=P + 512, qot=512), aq.EINVAL), (dict(qo=P + 128, qot=512), aq.EINVAL), (dict(qo=P), aq.EINVAL), (dict(qo=3 * P + 64), aq.EINVAL), (dict(qo=4 * P), aq.EINVAL),
    (dict(qo=2 * P), aq.EINVAL)])
def test_append(kw, code):
    assert _append(**kw) == code


def test_append_of_more_rows_than_a_launch_has_threads_for():
    """One head, T small enough for T Hkv <= 2^29: the limit stands between."""
    most = (1 << 30) // 12
    assert _append(T=most + 1, Hq=1, Hkv=1) == aq.ESHAPE
    assert _append(T=most, Hq=1, Hkv=1, slots=None) == aq.EINVAL


def test_append_without_rows():
    assert _append(T=0) == aq.OK and _append(T=0, k=None, v=None, q=None, qo=None, slots=None, pos=None) == aq.OK


@pytest.mark.parametrize("kw", [dict(dims=(3,)), dict(dims=()), dict(dims=(2, 2, 2, 2, 2)), dict(dims=(130,)), dict(dims=(0,)), dict(dims=(64,), layout="other"), dict(dims=(64,), freqs=[1.0]),
                                dict(dims=(4,), axis=[0, 1]), dict(dims=(4, -2))])
def test_tables_that_are_none(kw):
    with pytest.raises(aq.AttnQatError):
        aq.rope_table(**kw)


def test_a_table():
    r = aq.rope_table((4, 0, 2), theta=100.0)
    assert (r.pairs, r.axes, r.layout) == (3, 3, aq.ROPE_PAIRED) and r.axis[0] == 2 << 4
    for i, f in enumerate((1.0, 0.1, 1.0)):                        # (a frequency is within half a step of 53 bits)
        assert abs(r.turns[i] / 2.0 ** 64 - f / (2 * math.pi)) <= 2.0 ** -53


@pytest.mark.parametrize("f,turns", [(0.0, 0), (2 * math.pi, 0), (math.pi, 1 << 63), (-math.pi / 2, 3 << 62), (1e6, None), (-1e-30, None), (1e-12, None)])
def test_turns_of_a_frequency(f, turns):
    r = aq.rope_table((2,), freqs=[f])
    want = (Fraction(f) / PI2 % 1) * (1 << 64)
    assert abs((r.turns[0] - want + (1 << 63)) % (1 << 64) - (1 << 63)) <= 2 + abs(f) * 2.0      # (the quotient has 64 bits)
    if turns is not None:                                          # (pi of 53 bits)
        assert abs((r.turns[0] - turns + (1 << 63)) % (1 << 64) - (1 << 63)) <= 1 << 12


def _table(**kw):
    a = dict(rope=aq.Rope(), pairs=8, axes=2, layout=1, freq=[1.0] * 8, axis=[0, 1] * 4)
    a.update(kw)
    return aq.lib().attnqat_rope_table(None if a["rope"] is None else ctypes.addressof(a["rope"]), a["pairs"], a["axes"], a["layout"],
                                       None if a["freq"] is None else (ctypes.c_double * 65)(*a["freq"]), None if a["axis"] is None else (ctypes.c_uint8 * 65)(*a["axis"]))


@pytest.mark.parametrize("kw,code", [(dict(), aq.OK), (dict(rope=None), aq.EINVAL), (dict(freq=None), aq.EINVAL), (dict(axis=None), aq.EINVAL), (dict(pairs=0), aq.EINVAL), (dict(pairs=65), aq.EINVAL),
                                     (dict(axes=0), aq.EINVAL), (dict(axes=5), aq.EINVAL), (dict(layout=2), aq.EINVAL), (dict(axis=[0, 2]), aq.EINVAL), (dict(freq=[1.0, float("nan")]), aq.EINVAL),
                                     (dict(freq=[float("inf")]), aq.EINVAL), (dict(pairs=4), aq.ESHAPE), (dict(pairs=4, layout=0), aq.OK)])
def test_table_of_the_library(kw, code):
    assert _table(**kw) == code
