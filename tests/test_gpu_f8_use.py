"""Calls on scaled 8-bit floats, norms and experts as programs make them, on the GPU: captured in a graph with eager work between the replays; on
two streams at a time; on tensors that another stream made; with workspaces of their own; far into large tensors."""

import numpy as np
import pytest
import torch

from f8_ways import plan
from helpers import to_oracle
from oracle import f8
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def normal(shape, seed, dtype=BF):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def chosen(tokens, choices, experts, seed):
    return torch.randint(-1, experts, (tokens, choices), generator=torch.Generator().manual_seed(seed)).to(I32)


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


class Layer:
    """A norm, a product with shared sums, and experts with the gradient of their joining, on inputs that are written anew between calls."""

    def __init__(self, tokens, seed):
        width, hidden, experts = 4480, 300, 7
        self.x, self.residual, self.gain = (normal(s, seed + i).to(DEV) for i, s in enumerate(((tokens, width), (tokens, width), (width,))))
        self.w = gs.f8_quantize(normal((70, width), seed + 3).to(DEV), block_rows=128)
        self.up = gs.f8_quantize(normal((experts, hidden, width), seed + 4).to(DEV), block_rows=128)
        self.experts = chosen(tokens, 5, experts, seed + 5).to(DEV)
        self.weights = torch.rand(tokens, 5, generator=torch.Generator().manual_seed(seed + 6)).to(DEV)
        self.rows, self.grad_rows = (torch.zeros(tokens * 5, width if i else hidden, dtype=BF, device=DEV) for i in range(2))

    def __call__(self):
        y, total = gs.f8_norm(self.x, self.gain, residual=self.residual)
        z = gs.f8_dot(y, self.w)
        s = gs.expert_sort(self.experts, 7)
        self.rows.zero_()
        h = gs.f8_expert_dot(y, self.up, s.offsets, tokens=s.tokens, act=gs.GS_ACT_RELU, out=self.rows)
        j = gs.expert_join(h, s.places, self.weights)
        self.grad_rows.zero_()
        spread = gs.expert_split(total, s.places, out=self.grad_rows)
        grad = gs.expert_join_grad(total, spread, s.places, self.weights, grad_rows=torch.zeros_like(spread))
        return (y.values, y.scales, total, z, *s, h.clone(), j, spread.clone(), *grad, gs.norm(j)[0], gs.f8_dequantize(gs.f8_quantize(j)))

    def renew(self, seed):
        for i, t in enumerate((self.x, self.residual)):
            t.copy_(normal(tuple(t.shape), seed + i))
        self.experts.copy_(chosen(*self.experts.shape, 7, seed + 2))


@pytest.mark.parametrize("tokens", [18, 1100])
def test_captured_and_replayed(tokens):
    """Small ones: products with shared sums, a sort in one workgroup; many: several."""
    assert plan(18, 70, 4480, 0)[1] > 1 and gs.lib().glenside_expert_sort_workspace(1100 * 5, 7) > 0
    eager, graphed = Layer(tokens, 1), Layer(tokens, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = graphed()
    for i in range(4):
        eager.renew(100 + 10 * i)
        graphed.renew(100 + 10 * i)
        graph.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(got, want)):
            assert same(a, b), k


def test_two_graphs_at_a_time():
    """Graphs captured on different streams do not share a workspace: replayed together they give what each gives alone."""
    jobs, graphs, results = [Layer(1100, 20), Layer(1100, 40)], [], []
    want = [job() for job in jobs]
    for job in jobs:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(job())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for got, alone in zip(results, want):
            for a, b in zip(got, alone):
                assert same(a, b)


def test_two_streams_at_a_time():
    jobs = [Layer(18, 60), Layer(1100, 80)]
    alone = [job() for job in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(jobs[i]())
    torch.cuda.synchronize()
    for i in range(2):
        for results in got[i]:
            for a, b in zip(results, alone[i]):
                assert same(a, b)


def test_calls_go_to_the_current_stream():
    """On a stream that waits for the inputs' one, and back: a call on any other stream would not see them."""
    w = gs.f8_quantize(normal((4096, 4096), 1).to(DEV), block_rows=128)
    x = normal((300, 4096), 2).to(DEV)
    want = gs.f8_dot(gs.f8_norm(x)[0], w)
    torch.cuda.synchronize()
    for _ in range(5):
        side = torch.cuda.Stream()
        a = torch.zeros_like(x)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                a.copy_(x * 0.5)
            a.add_(a)
            got = gs.f8_dot(gs.f8_norm(a)[0], w)
            a.zero_()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        torch.cuda.synchronize()


def test_workspaces_given():
    (m, n, k), e = (18, 70, 4480), chosen(3000, 3, 20, 5).to(DEV)
    x, w = gs.f8_quantize(normal((m, k), 1).to(DEV)), gs.f8_quantize(normal((n, k), 2).to(DEV), block_rows=128)
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(gs.f8_dot(x, w, workspace=ws), gs.f8_dot(x, w))
    for a, b in zip(gs.expert_sort(e, 20, workspace=ws), gs.expert_sort(e, 20)):
        assert torch.equal(a, b)
    for call in (lambda t: gs.f8_dot(x, w, workspace=t), lambda t: gs.expert_sort(e, 20, workspace=t)):
        for short in (ws[:64], ws[8:]):
            with pytest.raises(gs.GlensideError) as err:
                call(short)
            assert err.value.status == gs.GS_ERR_WORKSPACE


def test_sorted_into():
    e = chosen(100, 3, 9, 1).to(DEV)
    out = gs.ExpertSort(*(torch.full((n,), 7, dtype=I32, device=DEV) for n in (10, 300)), torch.full((100, 3), 7, dtype=I32, device=DEV))
    assert gs.expert_sort(e, 9, out=out) is out
    for a, b in zip(out, gs.expert_sort(e, 9)):
        assert torch.equal(a, b)


def test_beyond_32_bits():
    """Offsets of bytes above 2^32: rows at the far end of matrices, of x read through an index, and of tokens spread out."""
    k, far = 8192, (1 << 19) + 300
    x = torch.zeros(far, k, dtype=BF, device=DEV)
    x[-3:] = normal((3, k), 1).to(DEV)
    m = gs.f8_quantize(x)                                                      # 4.3 GB of codes
    code, scales = f8.quantize(to_oracle(x[-3:])[None])
    assert np.array_equal(m.values[-3:].view(torch.uint8).cpu().numpy(), code[0]) and np.array_equal(to_oracle(m.scales[-3:]), scales[0])
    back = gs.f8_dequantize(m, out=torch.empty_like(x))
    assert np.array_equal(to_oracle(back[-3:].float()), to_oracle(torch.from_numpy(f8.round32(f8.dequantize(code, scales, k)[0])).to(BF)))
    y, _ = gs.norm(x, out=back)
    assert torch.equal(y[-3:], gs.norm(x[-3:].contiguous())[0])
    w = gs.f8_quantize(normal((130, k), 2).to(DEV), block_rows=128)
    want = gs.f8_dot(gs.F8(m.values[-3:].contiguous(), m.scales[-3:].contiguous(), (3, k), 1, 1), w)
    got = gs.f8_dot(m, w, out_dtype=BF)[-3:]
    assert (got.float() - want).abs().max() <= want.abs().max() * 2.0 ** -7
    # experts' rows: a few, and more than tiles take
    two = gs.F8(torch.stack((w.values, w.values)), torch.stack((w.scales, w.scales)), (2, 130, k), 2, 128)
    for rows in (6, 600):
        tokens = far - 1 - torch.arange(rows, dtype=I32, device=DEV) % 3
        got = gs.f8_expert_dot(m, two, torch.tensor([0, rows // 2, rows], dtype=I32, device=DEV), tokens=tokens)
        assert (got - want.flip(0).repeat(rows // 3, 1)).abs().max() <= want.abs().max() * 2.0 ** -12
    del m, back, y
    places = torch.full((3, 2), -1, dtype=I32, device=DEV)
    places[1, 1], places[2, 0] = far - 1, far - 2
    few = normal((3, k), 4).to(DEV)
    gs.expert_split(few, places, out=x)
    assert torch.equal(x[-1], few[1]) and torch.equal(x[-2], few[2])
    joined = gs.expert_join(x, places)
    assert torch.equal(joined[1:], few[1:]) and not joined[0].any()
    a, b = gs.expert_join_grad(few, x, places, grad_rows=x.clone())
    assert torch.equal(a[-1], few[1]) and b[1, 1] > 0 and b[0, 0] == 0
