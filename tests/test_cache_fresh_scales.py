"""CPU: the plain cache gives the pages that extend takes scale 0, so that a write that
leaves tokens of a page out takes nothing over from the page's last owner."""
import numpy as np

from oracle.cache import CacheOracle


def test_scales_of_a_recycled_page():
    o = CacheOracle(2, 3, 1, 2, 2, 2)
    assert o.extend([0], [70]) == 0
    big = np.full((70, 1, 2), 1e4)
    for layer in (0, 1):
        o.write(layer, [0, 70], [0], None, big, big, 1e38)
    o.free([0])
    assert o.extend([1], [60]) == 0 and o.table[1, 0] == 0
    assert not o.scale["k"][:, 0].any() and o.scale["v"][0, 1, 0] == 32.0
    x = np.random.default_rng(0).uniform(0.25, 0.5, (60, 1, 2))
    for at in (range(40), range(40, 60)):
        o.write(0, [0, len(at)], [1], list(at), x[list(at)], x[list(at)], 1e38)
    k, v = o.read(0, [0, 60], [1], None)
    assert (np.abs(k - x) <= x * 2.0 ** -4).all() and np.array_equal(k, v)
    assert o.extend([1], [5]) == 0 and o.scale["k"][0, 0, 0] == 2.0 ** -9 and o.scale["k"][0, 1, 0] == 0
