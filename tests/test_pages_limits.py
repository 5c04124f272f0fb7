"""The ends of what the rotary positions and attention over pages take, as the header states them."""
import pytest

from paper_2002_02645_amd import binding
from tests.test_pages_refusals import GB, P, at, pool

EINVAL = binding.FREEZE_EINVAL


@pytest.mark.parametrize("scale,taken", [(1e-38, True), (2e38, True), (2.01e38, False), (3e38, False), (0.0, False), (-1e-38, False)])
def test_scale(scale, taken):
    p = pool()
    got = binding.lib().freeze_pages_attend(at(p), 0, P(6 * GB), 1, 240, 40, 2, 0, None, 0, scale, 0, P(7 * GB), 1, 240, 40, P(8 * GB), GB, None)
    assert got == (0 if taken else EINVAL)


@pytest.mark.parametrize("factor,taken", [(3e38, True), (-3e38, True), (3.01e38, False), (-3.01e38, False)])
def test_factor(factor, taken):
    h = binding.FreezeHeads(GB, 2 * GB, 1, 3, 24, 8, 24, 8)
    assert binding.lib().freeze_rotate_positions(at(h), 1, 0, 8, P(8 * GB), P(9 * GB), 4, 0, factor, 0, None) == (0 if taken else EINVAL)
