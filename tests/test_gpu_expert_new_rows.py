"""Rows that are nobody's, in results that the binding makes: zeros, whatever the memory held; with a result given they stay as they were."""

import pytest
import torch

from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def soil(like):
    """Leaves memory of this tensor's size full of NaN behind, for the next one of the size to get."""
    torch.cuda.synchronize()
    full = torch.full_like(like, float("nan"))
    at = full.data_ptr()
    del full
    return at


def dealt(tokens, choices, experts, kept):
    """Sorted choices of which about `kept` of ten are some expert's."""
    g = torch.Generator().manual_seed(tokens + kept)
    e = torch.randint(0, experts, (tokens, choices), generator=g)
    e = torch.where(torch.randint(0, 10, (tokens, choices), generator=g) < kept, e, -1)
    return gs.expert_sort(e.to(I32).to(DEV), experts)


@pytest.mark.parametrize("kept", [0, 7, 10])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,choices,cols", [(1, 1, 1), (5, 2, 7), (100, 3, 264), (2000, 2, 130)])
def test_split_and_gradient(tokens, choices, cols, dtype, kept):
    s = dealt(tokens, choices, 6, kept)
    end, rows = int(s.offsets[-1]), normal((tokens * choices, cols), 1, dtype)
    x, weights = normal((tokens, cols), 2, dtype), normal((tokens, choices), 3, F32)
    given = gs.expert_split(x, s.places, out=torch.full_like(rows, 5.0))
    soil(rows)
    got = gs.expert_split(x, s.places)
    assert torch.equal(got[:end], given[:end]) and not got[end:].any() and (given[end:] == 5).all()
    given = gs.expert_join_grad(x, rows, s.places, weights, grad_rows=torch.full_like(rows, 5.0))
    soil(rows)
    got = gs.expert_join_grad(x, rows, s.places, weights)
    assert torch.equal(got[0][:end], given[0][:end]) and not got[0][end:].any() and (given[0][end:] == 5).all()
    assert torch.equal(got[1], given[1])


@pytest.mark.parametrize("dtype", [torch.int8, I32, torch.float8_e4m3fn])
def test_split_of_other_types(dtype):
    s = dealt(50, 2, 5, 7)
    end, x = int(s.offsets[-1]), (normal((50, 9), 1, F32) * 20).to(dtype)
    soil(torch.empty(100 * 9 * x.element_size() // 4, device=DEV))
    got = gs.expert_split(x, s.places)
    assert got.dtype == dtype and torch.equal(got.view(torch.uint8), gs.expert_split(x, s.places, out=torch.zeros_like(got)).view(torch.uint8))
    assert 0 < end < 100 and not got[end:].view(torch.uint8).any()


@pytest.mark.parametrize("kept", [0, 7, 10])
@pytest.mark.parametrize("tokens", [3, 900])
def test_products(tokens, kept):
    n, k = 70, 200
    s = dealt(tokens, 2, 5, kept)
    end = int(s.offsets[-1])
    x, w = gs.f8_quantize(normal((tokens, k), 1, BF)), gs.f8_quantize(normal((5, n, k), 2, BF), block_rows=128)
    for odt in (F32, BF):
        given = gs.f8_expert_dot(x, w, s.offsets, tokens=s.tokens, out=torch.full((tokens * 2, n), 5, dtype=odt, device=DEV))
        soil(given)
        got = gs.f8_expert_dot(x, w, s.offsets, tokens=s.tokens, out_dtype=odt)
        assert torch.equal(got[:end], given[:end]) and not got[end:].any() and (given[end:] == 5).all()


def test_captured():
    """The zeros are part of a captured call: every replay's rows that are nobody's are."""
    s, cols = dealt(60, 2, 5, 7), 130
    x = normal((60, cols), 1, BF)
    w = gs.f8_quantize(normal((5, 70, cols), 2, BF), block_rows=128)
    y = gs.f8_quantize(x)
    calls = (lambda: gs.expert_split(x, s.places), lambda: gs.expert_join_grad(x, rows, s.places)[0],
             lambda: gs.f8_expert_dot(y, w, s.offsets, tokens=s.tokens))
    rows = normal((120, cols), 3, BF)
    want = [call() for call in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for call in calls:
            call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [call() for call in calls]
    for i in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b) and not a[int(s.offsets[-1]):].any(), i
