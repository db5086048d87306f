"""What the entry points of a serving step refuse, by status and before anything is enqueued (no GPU is touched: the pointers are numbers)."""
import pytest

import paper_2603_00040_amd as aq

P = 1 << 20                                                       # some 16-byte aligned address that nobody follows


def _plan(**kw):
    a = dict(kv=P, new=2 * P, B=4, table=3 * P, max_pages=8, ring=4 * P, places=64, state=5 * P, T=16, kv_out=6 * P, cu=7 * P, slots=8 * P, pos=9 * P, state_out=10 * P,
             ws=11 * P, ws_bytes=1 << 16)
    a.update(kw)
    return aq.lib().attnqat_page_plan(a["kv"], a["new"], a["B"], a["table"], a["max_pages"], a["ring"], a["places"], a["state"], a["T"], a["kv_out"], a["cu"], a["slots"], a["pos"],
                                      a["state_out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(kv=None), aq.EINVAL), (dict(new=None), aq.EINVAL), (dict(table=None), aq.EINVAL), (dict(kv_out=None), aq.EINVAL), (dict(cu=None), aq.EINVAL),
    (dict(slots=None), aq.EINVAL), (dict(pos=None), aq.EINVAL), (dict(B=0), aq.EINVAL), (dict(max_pages=0), aq.EINVAL), (dict(T=-1), aq.EINVAL),
    (dict(places=0), aq.EINVAL), (dict(state=None), aq.EINVAL), (dict(state_out=None), aq.EINVAL), (dict(ring=None), aq.EINVAL), (dict(slots=8 * P + 4), aq.EINVAL),
    (dict(cu=P + 8), aq.EINVAL), (dict(cu=2 * P), aq.EINVAL), (dict(B=65536), aq.ESHAPE), (dict(max_pages=8193), aq.ESHAPE),
    (dict(ws=None), aq.EWORKSPACE), (dict(ws_bytes=16), aq.EWORKSPACE), (dict(ws=11 * P + 4), aq.EWORKSPACE)])
def test_plan(kw, code):
    assert _plan(**kw) == code


def _append(**kw):
    a = dict(k=P, kt=1024, kh=128, v=2 * P, vt=1024, vh=128, T=5, Hkv=8, d=128, dtype=0, cache=3 * P, pages=4, slots=4 * P)
    a.update(kw)
    L = aq.lib()
    return (L.attnqat_kv_cache_append(a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], a["T"], a["Hkv"], a["d"], a["dtype"], a["cache"], a["pages"], a["slots"], None),
            L.attnqat_kv_cache_read(a["cache"], a["pages"], a["slots"], a["T"], a["Hkv"], a["d"], a["dtype"], a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], None))


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), aq.EINVAL), (dict(v=None), aq.EINVAL), (dict(cache=None), aq.EINVAL), (dict(slots=None), aq.EINVAL), (dict(pages=0), aq.EINVAL), (dict(Hkv=0), aq.EINVAL),
    (dict(T=-1), aq.EINVAL), (dict(dtype=1), aq.EDTYPE), (dict(d=96), aq.ESHAPE), (dict(Hkv=1 << 29), aq.ESHAPE), (dict(T=(1 << 27) + 1), aq.ESHAPE), (dict(k=P + 8), aq.EINVAL), (dict(v=P + 2), aq.EINVAL),
    (dict(cache=3 * P + 8), aq.EINVAL), (dict(slots=4 * P + 4), aq.EINVAL), (dict(kt=1028), aq.EINVAL), (dict(vh=132), aq.EINVAL), (dict(kt=-1024), aq.EINVAL),
    (dict(vt=1 << 60), aq.EINVAL), (dict(kh=1 << 60), aq.EINVAL)])
def test_append_and_read(kw, code):
    assert _append(**kw) == (code, code)


@pytest.mark.parametrize("kw", [dict(kt=64), dict(vh=64), dict(kt=1016), dict(kt=0), dict(kh=0)])
def test_read_refuses_rows_that_overlap(kw):
    assert _append(**kw)[1] == aq.EINVAL


def test_no_rows_no_work():
    assert _append(T=0) == (aq.OK, aq.OK)
    assert _append(T=0, k=None, v=None, slots=None) == (aq.OK, aq.OK)
    assert _attend(T=0, q=None, o=None) == aq.OK


def _attend(**kw):
    a = dict(q=P, qt=1024, qh=128, cu=2 * P, T=5, max_q=3, B=2, Hq=8, Hkv=2, d=128, causal=1, window=0, scale=0.1, dtype=0, cache=3 * P, pages=4, table=4 * P, max_pages=8,
             lens=5 * P, o=6 * P, ot=1024, oh=128, lse=7 * P, ws=8 * P, ws_bytes=1 << 28)
    a.update(kw)
    return aq.lib().attnqat_fwd_kv4_ragged(a["q"], a["qt"], a["qh"], a["cu"], a["T"], a["max_q"], a["B"], a["Hq"], a["Hkv"], a["d"], a["causal"], a["window"], a["scale"], a["dtype"],
                                           a["cache"], a["pages"], a["table"], a["max_pages"], a["lens"], a["o"], a["ot"], a["oh"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), aq.EINVAL), (dict(cu=None), aq.EINVAL), (dict(cache=None), aq.EINVAL), (dict(table=None), aq.EINVAL), (dict(lens=None), aq.EINVAL), (dict(o=None), aq.EINVAL),
    (dict(T=-1), aq.EINVAL), (dict(max_q=0), aq.EINVAL), (dict(B=0), aq.EINVAL), (dict(Hq=0), aq.EINVAL), (dict(Hkv=0), aq.EINVAL), (dict(max_pages=0), aq.EINVAL),
    (dict(pages=0), aq.EINVAL), (dict(window=-1), aq.EINVAL), (dict(window=4, causal=0), aq.EINVAL), (dict(scale=0.0), aq.EINVAL), (dict(scale=-1.0), aq.EINVAL),
    (dict(scale=float("nan")), aq.EINVAL), (dict(scale=float("inf")), aq.EINVAL), (dict(d=32), aq.ESHAPE), (dict(Hkv=3), aq.ESHAPE), (dict(B=65536), aq.ESHAPE),
    (dict(max_pages=8193), aq.ESHAPE), (dict(T=1 << 26), aq.ESHAPE), (dict(dtype=2), aq.EDTYPE), (dict(q=P + 8), aq.EINVAL), (dict(o=6 * P + 8), aq.EINVAL),
    (dict(cache=3 * P + 8), aq.EINVAL), (dict(qt=1025), aq.EINVAL), (dict(oh=64), aq.EINVAL), (dict(ot=512), aq.EINVAL), (dict(o=P), aq.EINVAL), (dict(o=P + 1024), aq.EINVAL),
    (dict(lse=P), aq.EINVAL), (dict(lse=6 * P + 16), aq.EINVAL), (dict(ws=None), aq.EWORKSPACE), (dict(ws_bytes=0), aq.EWORKSPACE), (dict(ws=8 * P + 8), aq.EWORKSPACE)])
def test_attention(kw, code):
    assert _attend(**kw) == code


def test_size_queries():
    assert aq.page_plan_workspace_bytes(0) == 0 and aq.page_plan_workspace_bytes(65536) == 0
    assert aq.page_plan_workspace_bytes(100) >= 1600
    assert aq.kv4_ragged_workspace_bytes(0, 1, 8, 2, 1, 1, 128) > 0
    for bad in ((-1, 1, 8, 2, 1, 1, 128), (4, 0, 8, 2, 1, 1, 128), (4, 1, 8, 3, 1, 1, 128), (4, 1, 8, 2, 0, 1, 128), (4, 1, 8, 2, 1, 9000, 128), (4, 1, 8, 2, 1, 1, 80)):
        assert aq.kv4_ragged_workspace_bytes(*bad) == 0


def test_more_than_a_launch_holds():
    assert _plan(T=(1 << 29) + 1) == aq.ESHAPE
    assert _append(T=(1 << 26) + 1) == (aq.ESHAPE, aq.ESHAPE)
    assert _attend(B=65535, Hq=128, Hkv=128) == aq.ESHAPE and aq.kv4_ragged_workspace_bytes(4, 65535, 128, 128, 1, 1, 128) == 0


def test_plan_refuses_a_ring_that_lies_over_the_table():
    assert _plan(ring=3 * P + 64) == aq.EINVAL
