"""Products of scaled 8-bit floats in every way in which they are done, on small whole numbers with scales of powers of two: all sums are
exact in fp32 whatever their order, so results are compared bit for bit, and a number in a wrong place shows."""

import pytest
import torch

from f8_ways import WAYS
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def whole(shape, block_rows, seed):
    """An F8 pattern (mats, rows, K) and its numbers in float64; products of two of them are multiples of one and sums below 2^24."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    mats, rows, k = shape
    blocks, run = -(-k // 128), -(-k // 512) * 4
    codes = torch.randint(-3, 4, shape, generator=g, device=DEV).float()
    codes = torch.nn.functional.pad(codes, (0, blocks * 128 - k)).to(torch.float8_e4m3fn).view(mats, rows, blocks, 128)
    scales = torch.exp2(torch.randint(0, 3, (mats, -(-rows // block_rows), run), generator=g, device=DEV).float())
    of = torch.arange(rows, device=DEV) // block_rows
    return codes, scales, (codes.double() * scales[:, of, :blocks, None].double()).flatten(2)


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("way,splits,m,n,k,experts", [w for w in WAYS if w[5] == 0])
def test_one_matrix(way, splits, m, n, k, experts, w_rows):
    (xc, xs, xv), (wc, ws, wv) = whole((1, m, k), 1, m), whole((1, n, k), w_rows, n)
    x, w = gs.F8(xc[0], xs[0], (m, k), 1, 1), gs.F8(wc[0], ws[0], (n, k), 1, w_rows)
    want = xv[0] @ wv[0].t().contiguous()
    for odt in (F32, BF):
        store = torch.full((m * n + 64,), 7, dtype=odt, device=DEV)
        gs.f8_dot(x, w, out=store[:m * n].view(m, n))
        assert torch.equal(store[:m * n].view(m, n), want.float().to(odt)) and (store[m * n:] == 7).all()
    assert torch.equal(gs.f8_dot(x, w, act=gs.GS_ACT_RELU), want.clamp(min=0).float())


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("way,splits,m,n,k,experts", [w for w in WAYS if w[5] > 0])
def test_experts(way, splits, m, n, k, experts, w_rows, gather):
    (xc, xs, xv), (wc, ws, wv) = whole((1, m, k), 1, m), whole((experts, n, k), w_rows, n)
    g = torch.Generator().manual_seed(k)
    cuts = torch.sort(torch.randint(0, m + 1, (experts - 1,), generator=g)).values
    offsets = torch.cat((torch.tensor([0]), cuts, torch.tensor([m - 1 if m > 20 else m])))
    offsets = torch.cummax(offsets, 0).values
    tokens = torch.randint(-1, m, (m,), generator=g).to(I32).to(DEV) if gather else None
    x, w = gs.F8(xc[0], xs[0], (m, k), 1, 1), gs.F8(wc, ws, (experts, n, k), 2, w_rows)
    rows = xv[0] if not gather else torch.where((tokens >= 0).unsqueeze(1), xv[0][tokens.long().clamp(min=0)], 0.0)
    want = torch.full((m + 3, n), 5.0, dtype=torch.float64, device=DEV)
    for e in range(experts):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        want[lo:hi] = rows[lo:hi] @ wv[e].t().contiguous()
    for odt in (F32, BF):
        store = torch.full((m + 3, n), 5.0, dtype=odt, device=DEV)
        gs.f8_expert_dot(x, w, offsets.to(I32).to(DEV), tokens=tokens, out=store[:m])
        assert torch.equal(store, want.float().to(odt))
