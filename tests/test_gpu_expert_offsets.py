"""Experts' products with offsets in no order on the GPU: an offset below one before it counts as that one, so that no row is two experts', and
rows of no expert stay as they were.  Small whole numbers, whose sums are exact: results are compared bit for bit with the rule by hand."""

import pytest
import torch

from f8_ways import plan
from paper_2105_09377_amd import binding as gs
from test_gpu_f8_ways import DEV, F32, I32, whole

pytestmark = pytest.mark.gpu
TOP, LOW = 2 ** 31 - 1, -2 ** 31


def tables(rows, experts):
    """Offsets in no order: by hand where there are four experts, drawn and with what sorting could never give where there are more."""
    if experts == 4:
        half = rows // 2
        return [[0, half, 1, rows, 2], [rows, TOP, LOW, 3, 1], [half, 0, 0, half + 1, rows], [LOW, rows, 0, rows, 0], [0, 3, 2, 1, 0], [-5, 4, LOW, 5, TOP]]
    g = torch.Generator().manual_seed(experts)
    out = [torch.randint(0, rows + 1, (experts + 1,), generator=g).tolist()]               # soon at the end
    up = torch.sort(torch.randint(0, rows + 1, (experts + 1,), generator=g)).values
    out.append(torch.where(torch.rand(experts + 1, generator=g) < 0.3, up - rows // 3, up).tolist())
    up[63], up[64], up[-2], up[-1] = LOW, 0, LOW, 0                                         # (64 at a time are looked at)
    out.append(up.tolist())
    return out


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("rows,experts,way", [(12, 4, 0), (150, 4, 2), (3000, 4, 2), (90, 70, 0), (1200, 70, 2), (700, 64, 2), (5000, 200, 2)])
def test_offsets_in_no_order(rows, experts, way, w_rows):
    n, k = 70, 200
    assert plan(rows, n, k, experts)[0] == way
    (xc, xs, xv), (wc, ws, wv) = whole((1, rows, k), 1, rows), whole((experts, n, k), w_rows, experts)
    x, w = gs.F8(xc[0], xs[0], (rows, k), 1, 1), gs.F8(wc, ws, (experts, n, k), 2, w_rows)
    for offsets in tables(rows, experts):
        owner = [-1] * rows
        lo = min(max(offsets[0], 0), rows)
        for e in range(experts):
            hi = max(lo, min(offsets[e + 1], rows))
            owner[lo:hi] = [e] * (hi - lo)
            lo = hi
        owner = torch.tensor(owner, device=DEV)
        want = torch.full((rows, n), 9.0, dtype=torch.float64, device=DEV)
        for e in set(owner.tolist()) - {-1}:
            want[owner == e] = xv[0][owner == e] @ wv[e].t().contiguous()
        got = gs.f8_expert_dot(x, w, torch.tensor(offsets, dtype=torch.int64).to(I32).to(DEV), out=torch.full((rows, n), 9.0, dtype=F32, device=DEV))
        assert torch.equal(got, want.float()), offsets[:8]
