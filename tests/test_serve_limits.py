"""What a serving step's entry points refuse at the ends of their ranges (no GPU is touched: the pointers are numbers)."""
import pytest

import paper_2603_00040_amd as aq
from tests.test_serve_refusals import _attend


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38, 1e39])
def test_a_factor_that_is_infinite_in_powers_of_two(scale):
    """The exponents are taken to base 2: of scale log2 e = inf a score of zero would be a NaN."""
    assert _attend(scale=scale) == aq.EINVAL
