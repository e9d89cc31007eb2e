"""Sums of products of scaled 8-bit floats that workgroups share: every way in which the library does so, with every number of parts that it
chooses, has a size among those that run on the GPU."""

import math
import random

import pytest

from f8_parts import PARTS, slabs_of
from f8_ways import WAYS, plan


@pytest.mark.parametrize("way,splits,m,n,k,experts", PARTS)
def test_way(way, splits, m, n, k, experts):
    assert plan(m, n, k, experts) == (way, splits)


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def test_every_way_and_number_of_parts_has_a_size():
    """Of those met by sizes drawn from one up to beyond the largest that are of use."""
    rng, met = random.Random(1), {}
    for i in range(150000):
        m, n, k = spread(rng, 1, 1 << 15), spread(rng, 1, 1 << 16), spread(rng, 1, 1 << 17)
        met.setdefault(plan(m, n, k, 0), (m, n, k))
    for i in range(50000):
        e, m, n, k = spread(rng, 1, 4096), spread(rng, 1, 1 << 16), spread(rng, 1, 1 << 15), spread(rng, 1, 1 << 15)
        assert plan(m, n, k, e)[1] == 1
    sizes = {(way, splits) for way, splits, m, n, k, experts in WAYS + PARTS if experts == 0}
    assert set(met) <= sizes, {p: size for p, size in met.items() if p not in sizes}
    assert {p for p in met if p[1] > 1} == {(way, parts) for way in range(2, 9) for parts in (2, 4, 8)}


def test_parts_are_no_shorter_than_five_slabs():
    """Eight on average; what is dealt are fours, the last of them short."""
    rng, least = random.Random(2), 8
    for i in range(100000):
        m, n, k = spread(rng, 1, 1 << 14), spread(rng, 1, 1 << 14), spread(rng, 900, 1 << 15)
        parts = plan(m, n, k, 0)[1]
        each = slabs_of(k, parts)
        assert sum(each) == -(-k // 128) and all(n % 4 == 0 for n in each[:-1])
        if parts > 1:
            assert sum(each) >= 8 * parts
            least = min(least, *each)
    assert least == 5
