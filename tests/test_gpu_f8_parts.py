"""Products of scaled 8-bit floats whose sums workgroups share, in every way and number of parts, bit for bit as in test_gpu_f8_ways.py: sums of
these whole numbers stay below 144 K < 2^24."""

import pytest
import torch

from f8_parts import PARTS
from paper_2105_09377_amd import binding as gs
from test_gpu_f8_ways import BF, DEV, F32, whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("way,splits,m,n,k,experts", PARTS)
def test_one_matrix(way, splits, m, n, k, experts, w_rows):
    (xc, xs, xv), (wc, ws, wv) = whole((1, m, k), 1, m), whole((1, n, k), w_rows, n)
    x, w = gs.F8(xc[0], xs[0], (m, k), 1, 1), gs.F8(wc[0], ws[0], (n, k), 1, w_rows)
    want = xv[0] @ wv[0].t().contiguous()
    workspace = torch.full((splits * m * n * 4,), 255, dtype=torch.uint8, device=DEV)       # (NaN, were it added)
    for odt in (F32, BF):
        store = torch.full((m * n + 64,), 7, dtype=odt, device=DEV)
        gs.f8_dot(x, w, out=store[:m * n].view(m, n), workspace=workspace)
        assert torch.equal(store[:m * n].view(m, n), want.float().to(odt)) and (store[m * n:] == 7).all()
    assert torch.equal(gs.f8_dot(x, w, act=gs.GS_ACT_RELU), want.clamp(min=0).float())
    with pytest.raises(gs.GlensideError):
        gs.f8_dot(x, w, workspace=workspace[:-16])
