"""Which byte ranges norms refuse, without a GPU: nothing is launched by any call here."""

import pytest

from paper_2105_09377_amd import binding as gs
from test_abi_host import FAKE
from test_f8_host import at, f8, ref

VALUES, SCALES = 4 * 128, 4 * 16          # bytes of the codes and scales of (4, 64)


def codes(values=FAKE + (9 << 20), scales=FAKE + (10 << 20)):
    return f8((4, 64), 1, values=values, scales=scales)


@pytest.mark.parametrize("back", ["first", "last"])
def test_codes_and_scales_in_an_inputs_place(back):
    """From an input's first byte on, or up to it with their last 16."""
    L = gs.lib()
    x, residual, weight, total = at(1, (4, 64), 1), at(2, (4, 64), 1), at(3, (64,), 0), at(4, (4, 64), 1)
    for of in (x, residual, weight):
        for sum_ in (total, None):
            args = [ref(x), ref(residual), ref(weight), 1e-6, ref(sum_)]
            for onto in (codes(values=of.data - (VALUES - 16 if back == "last" else 0)), codes(scales=of.data - (SCALES - 16 if back == "last" else 0))):
                assert L.glenside_f8_norm(*args, ref(onto), None) == gs.GS_ERR_UNSUPPORTED
