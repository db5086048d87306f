"""Numbers that an int does not hold, in the Python calls of attention over chosen pages (CPU: none of these reaches the library)."""
import pytest
import torch

import paper_2603_00040_amd as aq


@pytest.mark.parametrize("pages", [0, -1, -4, 4 - (1 << 32), 4 + (1 << 32), -(1 << 63)])
def test_pages_of_a_summary(pages):
    """ctypes would take the low 32 bits: 4 of 4 - 2^32."""
    summary = torch.zeros(3 * 2 * (64 + 16), dtype=torch.uint8)
    with pytest.raises(aq.AttnQatError):
        aq._summary_pages(summary, pages, 2, 64)


def test_pages_that_a_summary_has_room_for():
    summary = torch.zeros(3 * 2 * (64 + 16), dtype=torch.uint8)
    for pages in (1, 2, 3):
        aq._summary_pages(summary, pages, 2, 64)
    with pytest.raises(aq.AttnQatError):
        aq._summary_pages(summary, 4, 2, 64)
