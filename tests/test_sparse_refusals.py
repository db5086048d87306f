"""What the entry points of attention over chosen pages refuse, by status and before anything is enqueued (no GPU is touched: the pointers are numbers)."""
import pytest

import paper_2603_00040_amd as aq

P = 1 << 24


def _summarize(**kw):
    a = dict(cache=P, pages=4, slots=2 * P, T=5, Hkv=2, d=128, summary=3 * P)
    a.update(kw)
    return aq.lib().attnqat_kv_summarize(a["cache"], a["pages"], a["slots"], a["T"], a["Hkv"], a["d"], a["summary"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), aq.EINVAL), (dict(slots=None), aq.EINVAL), (dict(summary=None), aq.EINVAL), (dict(pages=0), aq.EINVAL), (dict(T=-1), aq.EINVAL), (dict(Hkv=0), aq.EINVAL),
    (dict(d=32), aq.ESHAPE), (dict(T=(1 << 29) + 1), aq.ESHAPE), (dict(Hkv=65536), aq.ESHAPE), (dict(cache=P + 8), aq.EINVAL), (dict(slots=2 * P + 4), aq.EINVAL),
    (dict(summary=3 * P + 8), aq.EINVAL), (dict(summary=P + 1024), aq.EINVAL), (dict(summary=2 * P - 16), aq.EINVAL)])
def test_summarize(kw, code):
    assert _summarize(**kw) == code


def _select(**kw):
    a = dict(q=P, qt=1024, qh=128, cu=2 * P, T=5, max_q=3, B=2, Hq=8, Hkv=2, d=128, dtype=0, summary=3 * P, pages=4, table=4 * P, max_pages=8, lens=5 * P, n=6, first=1, last=1, blocks=6 * P)
    a.update(kw)
    return aq.lib().attnqat_kv_select(a["q"], a["qt"], a["qh"], a["cu"], a["T"], a["max_q"], a["B"], a["Hq"], a["Hkv"], a["d"], a["dtype"], a["summary"], a["pages"], a["table"],
                                      a["max_pages"], a["lens"], a["n"], a["first"], a["last"], a["blocks"], None)


STEP = [(dict(q=None), aq.EINVAL), (dict(cu=None), aq.EINVAL), (dict(table=None), aq.EINVAL), (dict(lens=None), aq.EINVAL), (dict(blocks=None), aq.EINVAL), (dict(T=-1), aq.EINVAL),
        (dict(max_q=0), aq.EINVAL), (dict(B=0), aq.EINVAL), (dict(Hq=0), aq.EINVAL), (dict(Hkv=0), aq.EINVAL), (dict(max_pages=0), aq.EINVAL), (dict(pages=0), aq.EINVAL),
        (dict(n=0), aq.EINVAL), (dict(d=32), aq.ESHAPE), (dict(Hkv=3), aq.ESHAPE), (dict(B=65536), aq.ESHAPE), (dict(max_pages=8193), aq.ESHAPE), (dict(n=1025), aq.ESHAPE),
        (dict(T=1 << 26), aq.ESHAPE), (dict(T=(1 << 22) + 1), aq.ESHAPE), (dict(dtype=2), aq.EDTYPE), (dict(q=P + 8), aq.EINVAL), (dict(qt=1025), aq.EINVAL), (dict(blocks=6 * P + 2), aq.EINVAL),
        (dict(blocks=P + 1024), aq.EINVAL)]


@pytest.mark.parametrize("kw,code", STEP + [
    (dict(summary=None), aq.EINVAL), (dict(summary=3 * P + 8), aq.EINVAL), (dict(first=-1), aq.EINVAL), (dict(last=0), aq.EINVAL), (dict(first=6), aq.EINVAL), (dict(last=7), aq.EINVAL),
    (dict(first=2147483647, last=2147483647), aq.EINVAL), (dict(blocks=3 * P), aq.EINVAL), (dict(blocks=4 * P), aq.EINVAL), (dict(blocks=5 * P), aq.EINVAL), (dict(blocks=2 * P), aq.EINVAL)])
def test_select(kw, code):
    assert _select(**kw) == code


def _attend(**kw):
    a = dict(q=P, qt=1024, qh=128, cu=2 * P, T=5, max_q=3, B=2, Hq=8, Hkv=2, d=128, scale=0.1, dtype=0, cache=3 * P, pages=4, table=4 * P, max_pages=8, lens=5 * P, blocks=6 * P, n=6,
             o=7 * P, ot=1024, oh=128, lse=8 * P, ws=9 * P, ws_bytes=1 << 28)
    a.update(kw)
    return aq.lib().attnqat_fwd_kv4_sparse(a["q"], a["qt"], a["qh"], a["cu"], a["T"], a["max_q"], a["B"], a["Hq"], a["Hkv"], a["d"], a["scale"], a["dtype"], a["cache"], a["pages"], a["table"],
                                           a["max_pages"], a["lens"], a["blocks"], a["n"], a["o"], a["ot"], a["oh"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [x for x in STEP if x[0] != dict(blocks=P + 1024)] + [
    (dict(cache=None), aq.EINVAL), (dict(o=None), aq.EINVAL), (dict(scale=0.0), aq.EINVAL), (dict(scale=-1.0), aq.EINVAL), (dict(scale=float("nan")), aq.EINVAL),
    (dict(scale=float("inf")), aq.EINVAL), (dict(scale=3e38), aq.EINVAL), (dict(o=7 * P + 8), aq.EINVAL), (dict(cache=3 * P + 8), aq.EINVAL), (dict(oh=64), aq.EINVAL), (dict(ot=512), aq.EINVAL),
    (dict(o=P), aq.EINVAL), (dict(o=P + 1024), aq.EINVAL), (dict(o=6 * P), aq.EINVAL), (dict(lse=P), aq.EINVAL), (dict(lse=7 * P + 16), aq.EINVAL), (dict(lse=6 * P), aq.EINVAL),
    (dict(ws=None), aq.EWORKSPACE), (dict(ws_bytes=0), aq.EWORKSPACE), (dict(ws=9 * P + 8), aq.EWORKSPACE)])
def test_attention(kw, code):
    assert _attend(**kw) == code


def test_no_rows_no_work():
    assert _summarize(T=0) == _select(T=0) == _attend(T=0) == aq.OK
    assert _summarize(T=0, slots=None) == _select(T=0, q=None, blocks=None) == _attend(T=0, q=None, o=None, blocks=None) == aq.OK


def test_size_queries():
    assert aq.kv_summary_page_bytes(8, 128) == 8 * 144 and aq.kv_summary_page_bytes(3, 64) == 240
    assert aq.kv_summary_page_bytes(0, 128) == aq.kv_summary_page_bytes(2, 96) == 0
    assert aq.kv4_sparse_workspace_bytes(0, 8, 2, 1, 4, 128) > 0
    few, many = aq.kv4_sparse_workspace_bytes(1, 8, 2, 1, 32, 128), aq.kv4_sparse_workspace_bytes(9000, 8, 2, 300, 32, 128)
    assert few > many > 0                                          # (pages are split where there are few rows)
    for bad in ((-1, 8, 2, 1, 4, 128), (4, 8, 3, 1, 4, 128), (4, 8, 2, 0, 4, 128), (4, 8, 2, 1, 0, 128), (4, 8, 2, 1, 1025, 128), (4, 8, 2, 1, 4, 80), (1 << 23, 8, 2, 1, 4, 128)):
        assert aq.kv4_sparse_workspace_bytes(*bad) == 0
