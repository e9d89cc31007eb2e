"""The oracle's experts' products with offsets in no order, against the rule by hand: an offset below one before it counts as that one, so that no
row is two experts', and rows of no expert stay as they were."""

import numpy as np
import pytest

from oracle import f8


@pytest.mark.parametrize("offsets,owner", [
    ([0, 2, 3, 5], [0, 0, 1, 2, 2, -1]), ([0, 4, 2, 5], [0, 0, 0, 0, 2, -1]), ([3, 1, 2, 6], [-1, -1, -1, 2, 2, 2]), ([6, 2 ** 31 - 1, -2 ** 31, 3], [-1] * 6),
    ([5, 1, 0, 0], [-1] * 6), ([-4, 6, 0, 6], [0] * 6), ([2, -1, 4, 3], [-1, -1, 1, 1, -1, -1])])
def test_offsets_in_no_order(offsets, owner):
    g = np.random.default_rng(1)
    x, w = g.integers(-3, 4, (6, 5)).astype(np.float64), g.integers(-3, 4, (3, 2, 5)).astype(np.float64)
    out, _ = f8.expert_dot(x, None, offsets, w, np.full((6, 2), 9.0))
    want = np.array([w[e] @ x[r] if e >= 0 else [9.0, 9.0] for r, e in enumerate(owner)])
    assert np.array_equal(out, want)
