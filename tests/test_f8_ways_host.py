"""The sizes of f8_ways.py are done in the ways that they stand for, and no way is without one."""

import pytest

from f8_ways import WAYS, plan


@pytest.mark.parametrize("way,splits,m,n,k,experts", WAYS)
def test_way(way, splits, m, n, k, experts):
    assert plan(m, n, k, experts) == (way, splits)


def test_every_way_has_a_size():
    for some in (False, True):
        assert {w[0] for w in WAYS if (w[5] > 0) == some} == set(range(9))
    assert {w[1] for w in WAYS} == {1, 2, 4}


def test_plans_of_many_sizes():
    """Sums of experts are never shared, nor short ones; workspaces are asked for exactly there."""
    for m in (0, 1, 5, 16, 17, 33, 100, 500, 3000, 70000):
        for n in (1, 50, 1000, 9000, 200000):
            for k in (0, 1, 128, 1000, 4096, 9000, 100000):
                way, splits = plan(m, n, k, 0)
                assert 0 <= way < 9 and (splits == 1 or (k + 127) // 128 >= 8 * splits)
                assert plan(m, n, k, 7)[1] == 1
