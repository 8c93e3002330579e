"""The inputs and bounds with which attention is tested on the device: that what a kernel could lose is outside of them (a mistake planted in the reference)."""
import pytest

from kv_plain import Batch
from kv_tight import Counted

SIZES = [[(1, 5000)], [(2, 3000), (1, 9)], [(3, 200)]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("dim", [64, 128])
def test_each_lost_key_shows(sizes, dim):
    c = Counted(Batch(sizes, 64, 1, dim, seed=1), 2)
    want = c.expected()
    length = int(c.b.lengths[0])
    for lost in [[0], [1], [length // 2], [length - 3], [length // 3, length // 3 + 1]]:
        assert ((c.expected(lost=lost) - want).abs() > c.bound(want))[0].any(), lost


@pytest.mark.parametrize("sizes", SIZES[:1])
def test_half_a_tile_shows(sizes):
    c = Counted(Batch(sizes, 64, 1, 128, seed=1), 2)
    want = c.expected()
    for first in (0, 128, 4960):
        assert ((c.expected(lost=range(first, first + 32)) - want).abs() > c.bound(want))[0].float().mean() > 0.2
