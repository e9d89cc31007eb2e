"""What the comparison of the 4-bit decoder stack with its definition can tell, without a GPU: each mistake planted in the definition lies
beyond what is allowed, wherever it changes anything."""

import pytest

import decoder4_reference as ref
from helpers import to_oracle

# (where it cannot change anything: no window, one layer, nothing quantised or all of it)
VOID = {"no window": lambda n, w, q: not w, "no sinks": lambda n, w, q: not w, "sinks one too few": lambda n, w, q: not w,
        "window one too long": lambda n, w, q: not w, "no quantising": lambda n, w, q: not q, "quantising all the same": lambda n, w, q: q,
        "one cache for both layers": lambda n, w, q: n == 1}


@pytest.mark.parametrize("n,window,sinks,quantize", ref.STACKS)
def test_mistakes_are_beyond_what_is_allowed(n, window, sinks, quantize):
    x = to_oracle(ref.tokens(2)[0])
    want, limit = ref.stack(n, x, window, sinks, quantize), ref.allowed(x, n, window, sinks, quantize)
    for mistake in ref.MISTAKES:
        off = ref.off(ref.stack(n, x, window, sinks, quantize, mistake), want, x)
        if VOID.get(mistake, lambda *_: False)(n, window, quantize):
            assert off == 0, mistake
        else:
            assert off > 1.5 * limit, (mistake, off, limit)
