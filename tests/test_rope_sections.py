"""Tables of rotary positions whose axes share one ladder of frequencies over the head, and those that begin it anew in every axis (CPU)."""
import paper_2603_00040_amd as aq


def _axis(r, i):
    return r.axis[i // 16] >> (2 * (i % 16)) & 3


def test_one_ladder_in_sections():
    """freqs alone: the sections are those of dims."""
    whole = aq.rope_table((128,), theta=1e6, layout="halves")
    r = aq.rope_table((32, 48, 48), layout="halves", freqs=[1e6 ** (-2.0 * i / 128) for i in range(64)])
    assert (r.pairs, r.axes, r.layout) == (64, 3, aq.ROPE_HALVES) and list(r.turns) == list(whole.turns)
    assert [_axis(r, i) for i in range(64)] == [0] * 16 + [1] * 24 + [2] * 24


def test_a_ladder_in_every_axis():
    r = aq.rope_table((32, 48, 48), theta=1e6, layout="halves")
    assert list(r.turns[:16]) == list(aq.rope_table((32,), theta=1e6, layout="halves").turns[:16])
    assert list(r.turns[16:40]) == list(r.turns[40:64]) == list(aq.rope_table((48,), theta=1e6, layout="halves").turns[:24])


def test_axes_in_turns():
    """axis alone: the frequencies are those of dims."""
    r = aq.rope_table((32, 32), axis=[0, 1] * 16)
    assert list(r.turns) == list(aq.rope_table((32, 32)).turns) and [_axis(r, i) for i in range(32)] == [0, 1] * 16
