"""What the comparison of the 8-bit decoder stack with its definition can tell, without a GPU: each mistake planted in the definition lies beyond
what is allowed, wherever it changes anything."""

import pytest

import decoder8_reference as ref
from helpers import to_oracle

# (with one layer there is no other cache, no layer before, and nothing to add to the first norm)
ONE = ("one cache for both layers", "the norm of the layer before", "residual not added")


@pytest.mark.parametrize("n", [1, 2])
def test_mistakes_are_beyond_what_is_allowed(n):
    x = to_oracle(ref.tokens(2)[0])
    want, limit = ref.stack(n, x, 0, 2), ref.allowed(x, n, 0, 2)
    assert limit < 0.07 * n
    for mistake in ref.MISTAKES:
        off = ref.off(ref.stack(n, x, 0, 2, mistake), want, x)
        if n == 1 and mistake in ONE:
            assert off == 0, mistake
        elif n == 2 and mistake == "no quantising":
            continue                         # (as much as codes on the other side do in two layers; it shows in one)
        else:
            assert off > 1.5 * limit, (mistake, off, limit)
