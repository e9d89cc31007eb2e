"""What a decoder layer's calls give a token, bit for bit the same whether it comes alone or among others, where the calls are done in the same way;
and so the whole stack's results."""

import pytest
import torch

import decoder8_reference as ref
from f8_ways import plan
from paper_2105_09377_amd import binding as gs
from test_gpu_decoder8 import BATCH, DEV, TABLE, Routes, run, stack

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_calls():
    """Norms, products, experts and their joining of twelve rows, and of the same ones in pieces; products of up to 16 rows, 8 to an expert, go through
    registers whatever their number."""
    w = {name: t.to(DEV) for name, t in ref.layers(1)[0].items()}
    dense, up = gs.f8_quantize(w["q"], block_rows=128), gs.f8_quantize(w["up"], block_rows=128)
    assert all(plan(m, dense.shape[0], ref.WIDTH, 0) == (0, 1) and plan(2 * m, ref.HIDDEN, ref.WIDTH, ref.EXPERTS) == (0, 1) for m in range(1, 13))
    x, residual = ref.tokens(BATCH).to(DEV)[:, :6].reshape(12, -1), ref.tokens(BATCH).to(DEV)[:, 6:12].reshape(12, -1)
    experts, weights = (t[:, :6].reshape(12, -1).to(DEV) for t in ref.routing(0, BATCH))

    def layer(rows):
        y, total = gs.f8_norm(x[rows], w["norm_attention"], residual=residual[rows])
        s = gs.expert_sort(experts[rows].clone(), ref.EXPERTS)
        h = gs.f8_expert_dot(y, up, s.offsets, tokens=s.tokens, out_dtype=BF, act=gs.GS_ACT_RELU)
        return y.values.view(torch.uint8), y.scales, total, gs.f8_dot(y, dense, out_dtype=BF), gs.expert_join(h, s.places, weights[rows].clone())

    together = layer(slice(0, 12))
    for pieces in ((1,) * 12, (5, 1, 6), (2, 3, 7)):
        at, parts = 0, []
        for n in pieces:
            parts.append(layer(slice(at, at + n)))
            at += n
        for i, want in enumerate(together):
            assert torch.equal(torch.cat([p[i] for p in parts]), want), (pieces, i)


@pytest.mark.parametrize("pieces", [(1, 2, 3), (1,) * 6])
def test_stack(pieces):
    """Two sequences of six tokens: twelve rows at most, attention over a few tokens in one part."""
    whole, parts = Routes(), Routes()
    x = ref.tokens(BATCH).to(DEV)[:, :6].contiguous()
    a = run(stack(2, whole), whole, x, (6,), TABLE.to(DEV))
    assert torch.equal(run(stack(2, parts), parts, x, pieces, TABLE.to(DEV)), a)
