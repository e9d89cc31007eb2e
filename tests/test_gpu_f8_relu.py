"""ReLU behind products of scaled 8-bit floats: zero of what is below zero, and of NaN, in every kernel that ends a product; without it a block whose
scale is NaN shows in its row, and in its row alone."""

import pytest
import torch

from f8_ways import plan
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF)


@pytest.mark.parametrize("odt", [F32, BF])
@pytest.mark.parametrize("m,n,k,way,parts", [(3, 40, 300, 0, 1), (40, 100, 900, 2, 1), (20, 70, 2922, 2, 2), (300, 4096, 4096, 4, 1)])
def test_one_matrix(m, n, k, way, parts, odt):
    assert plan(m, n, k, 0) == (way, parts)
    x = normal((m, k), 1)
    x[m // 2, k - 1] = float("inf")
    x, w = gs.f8_quantize(x.to(DEV)), gs.f8_quantize(normal((n, k), 2).to(DEV), block_rows=128)
    plain = gs.f8_dot(x, w, out_dtype=odt)
    assert torch.equal(torch.isnan(plain), (torch.arange(m, device=DEV) == m // 2).unsqueeze(1).expand(m, n))
    assert torch.equal(gs.f8_dot(x, w, out_dtype=odt, act=gs.GS_ACT_RELU), plain.nan_to_num(nan=0.0).clamp(min=0))


@pytest.mark.parametrize("rows", [8, 400])
def test_experts(rows):
    k, n = 200, 70
    x = normal((rows, k), 1)
    x[2, 3] = float("nan")
    x, w = gs.f8_quantize(x.to(DEV)), gs.f8_quantize(normal((2, n, k), 2).to(DEV), block_rows=128)
    offsets = torch.tensor([0, rows // 2, rows], dtype=I32, device=DEV)
    plain = gs.f8_expert_dot(x, w, offsets)
    assert torch.isnan(plain[2]).all() and torch.isnan(plain).sum() == n
    assert torch.equal(gs.f8_expert_dot(x, w, offsets, act=gs.GS_ACT_RELU), plain.nan_to_num(nan=0.0).clamp(min=0))
