"""A product goes out in two launches only where their cost is clearly less than one launch's (host code, no GPU)."""
import pytest

import host_shim
from test_gpu_quant import CUT_SIZES
from test_quant_choice import SHIM, plan


@pytest.fixture(scope="module")
def rule():
    return host_shim.build(SHIM)


def costs(rule, rows, cols, inner, n_cus=256):
    """One launch's cost, the chosen plan's (None for one launch)."""

    def rounds(i, n):
        return -(-(-(-rows // rule.tile(i, 0)) * -(-n // rule.tile(i, 1))) // n_cus) * rule.tile(i, 2)

    t, first, rest = plan(rule, rows, cols, inner, n_cus)
    one = rounds(rule.choice(rows, cols, n_cus), cols) * inner
    return one, None if first == cols else (rounds(t, first) + rounds(rest, cols - first) + 50) * inner + 40 * 4096


def test_sizes_that_two_launches_would_slow_down(rule):
    for rows, cols, inner in ((1500, 4096, 11008), (300, 22016, 4096), (350, 22016, 4096), (700, 11008, 5120), (800, 22016, 4096)):
        assert costs(rule, rows, cols, inner)[1] is None, (rows, cols, inner)


def test_two_launches_cost_clearly_less(rule):
    """By 50 for each value of the inner length, a fourteenth of a round of the largest tiles, and 40 at 4096."""
    cut = 0
    for rows in (129, 160, 300, 350, 512, 700, 1024, 1500, 2500, 4096, 8192):
        for cols in (4096, 5120, 8192, 11008, 12288, 13824, 15360, 22016, 27648, 32000):
            for inner in (256, 1024, 4096, 5120, 11008, 13824):
                one, two = costs(rule, rows, cols, inner)
                cut += two is not None
                assert two is None or two < one, (rows, cols, inner)
    assert cut > 20
    for size in CUT_SIZES:
        assert costs(rule, *size)[1] is not None
