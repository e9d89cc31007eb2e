"""Results that share bytes with each other are refused by norms and the calls on tokens, without a GPU: nothing is launched by any call here."""

from paper_2105_09377_amd import binding as gs
from test_abi_host import FAKE, ap
from test_f8_host import F32, I32, at, f8, ref


def test_norms():
    """The sum in the place of the norm, its codes or its scales; the codes' last bytes in that of the scales."""
    L, no = gs.lib(), gs.GS_ERR_UNSUPPORTED
    x, total = at(1, (4, 64), 1), at(4, (4, 64), 1)
    args = [ref(x), None, None, 1e-6, ref(total)]
    for back in (0, 4 * 64 * 2 - 16):
        assert L.glenside_norm(*args, ref(ap((4, 64), 1, data=total.data - back)), None) == no
    far = FAKE + (9 << 20)
    for codes in (f8((4, 64), 1, values=total.data, scales=far), f8((4, 64), 1, values=far, scales=total.data + 496), f8((4, 64), 1, values=far, scales=far + 496)):
        assert L.glenside_f8_norm(*args, ref(codes), None) == no
        if codes.scales == far + 496:
            assert L.glenside_f8_norm(*args[:4], None, ref(codes), None) == no


def test_calls_on_tokens():
    L, no = gs.lib(), gs.GS_ERR_UNSUPPORTED
    experts, offsets, tokens, places = at(1, (10, 3), 2, I32), at(2, (5,), 1, I32), at(3, (30,), 1, I32), at(4, (10, 3), 2, I32)
    for three in ((offsets, ap((30,), 1, I32, data=offsets.data), places), (offsets, tokens, ap((10, 3), 2, I32, data=tokens.data + 112)),
                  (ap((5,), 1, I32, data=places.data), tokens, places)):
        assert L.glenside_expert_sort(ref(experts), *(ref(t) for t in three), None, 0, None) == no
    flat, rows, places, weights, grad_rows = at(1, (10, 40), 1), at(2, (30, 40), 1), at(4, (10, 3), 2, I32), at(5, (10, 3), 2, F32), at(6, (30, 40), 1)
    for of in (grad_rows.data, grad_rows.data + 30 * 40 * 2 - 16):
        assert L.glenside_expert_join_grad(ref(flat), ref(rows), ref(places), ref(weights), ref(grad_rows), ref(ap((10, 3), 2, F32, data=of)), None) == no
