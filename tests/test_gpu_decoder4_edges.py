"""The stack of 4-bit decoder layers where a call has little or nothing to do."""

import pytest
import torch

from paper_2105_09377_amd import decoder4, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("quantize", [None, 0])
@pytest.mark.parametrize("batch,tokens", [(0, 3), (2, 0)])
def test_no_tokens(batch, tokens, quantize):
    shapes = decoder4.weight_shapes(64, 2, 1, 64, 96)
    layers = [{name: synth.normal_bf16(shape, 0.1, 9300 + i) for i, (name, shape) in enumerate(shapes.items())}]
    st = decoder4.Decoder4Stack(layers, 2, 1, 64, n_pages=4, page_size=16, quantize_rows=quantize, device=DEV)
    first = torch.zeros(batch, dtype=torch.int32, device=DEV)
    x = torch.zeros(batch, tokens, 64, dtype=torch.bfloat16, device=DEV)
    y = st.step(x, torch.zeros(batch, 2, dtype=torch.int32, device=DEV), first, first)
    assert y.shape == x.shape and y.dtype == x.dtype and not st.caches[0].data.any()
