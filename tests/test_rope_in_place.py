"""Rotary positions in place: an output may be its own input with the same strides, and only so.  Where two extents are equal, an output that has the input's elements in another
order (strides exchanged) is refused: its threads would write what others have yet to read.  By status, before anything is enqueued (no GPU is touched: the pointers are numbers)."""
import pytest

import paper_2603_00040_amd as aq
from tests.test_rope_refusals import P, _append, _call

accepted = pytest.mark.skipif(aq.torch.cuda.is_available(), reason="calls that are accepted would be enqueued")


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("B,H,L,src,dst", [
    (1, 16, 16, (0, 1024, 64), (0, 64, 1024)),                    # heads and tokens
    (2, 16, 16, (16384, 64, 1024), (16384, 1024, 64)),
    (16, 16, 3, (3072, 192, 64), (192, 3072, 64)),                # batches and heads
    (8, 4, 8, (2048, 512, 64), (64, 512, 2048)),                  # batches and tokens
    (3, 3, 3, (576, 192, 64), (192, 64, 576))])
def test_strides_exchanged(B, H, L, src, dst, back):
    kw = dict(B=B, Hq=H, Hkv=0, L=L, q=P, qs=src, qo=P, qos=dst, k=None, ko=None)
    assert _call(back, **kw) == aq.EINVAL
    kw.update(Hkv=H, k=P, ks=src, ko=P, kos=dst, q=3 * P, qo=4 * P)
    assert _call(back, **kw) == aq.EINVAL


def test_strides_exchanged_on_the_way_into_the_cache():
    assert _append(T=6, Hq=6, q=P, qt=384, qh=64, qo=P, qot=64, qoh=384, k=6 * P, v=7 * P) == aq.EINVAL


# Accepted: what is left to say is that no kernel can be launched here.
@accepted
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("B,H,L,src,dst", [
    (2, 16, 16, (16384, 64, 1024), (16384, 64, 1024)),
    (1, 16, 16, (0, 64, 1024), (7, 64, 1024)),                    # (no second batch, head or token: its stride says nothing)
    (2, 1, 16, (16384, 0, 1024), (16384, 3, 1024)),
    (2, 16, 1, (16384, 64, 5), (16384, 64, 1024)),
    (1, 1, 1, (0, 0, 0), (9, 9, 9))])
def test_in_place(B, H, L, src, dst, back):
    assert _call(back, B=B, Hq=H, Hkv=0, L=L, q=P, qs=src, qo=P, qos=dst, k=None, ko=None) == aq.ELAUNCH
    assert _call(back, B=B, Hq=H, Hkv=H, L=L, q=3 * P, qs=src, qo=4 * P, qos=dst, k=P, ks=src, ko=P, kos=dst) == aq.ELAUNCH


@accepted
def test_in_place_on_the_way_into_the_cache():
    assert _append(T=6, Hq=6, q=P, qt=384, qh=64, qo=P, qot=384, qoh=64, k=6 * P, v=7 * P) == aq.ELAUNCH
    assert _append(T=1, Hq=6, q=P, qt=8, qh=64, qo=P, qot=384, qoh=64, k=6 * P, v=7 * P) == aq.ELAUNCH
