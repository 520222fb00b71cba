"""Scales at their ends.  (Tolerances as in paged_util.)"""
import pytest

from paged_util import Cache, check

pytestmark = pytest.mark.gpu

FORMS = [(1, 1, 16, None), (1, 4, 16, None), (1, 4, 16, 3000), (4, 4, 7, 3000), (5, 4, 24, None), (5, 8, 24, 3000), (5, 8, 16, 3000),
         (2, 50, 64, 3000)]


@pytest.mark.parametrize("rows,group,page_rows,cols", FORMS)
def test_tiny_scales_of_huge_scores(rows, group, page_rows, cols):
    """Keys of 2^110: their products are numbers, and so is the scale that brings them down to ordinary scores."""
    c = Cache([700, 3000, 40], rows, 2 * group, 2, 64, "bf16", page_rows, cols=cols, seed=rows + 1)
    for i in range(3):
        c.keys[i] = c.keys[i] * 2.0 ** 110
        c.put(i, 0, c.keys[i], c.values[i])
    check(c, scale=2.0 ** -113)
    check(c, scale=0.0)
