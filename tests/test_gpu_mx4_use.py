"""Calls on microscaled 4-bit floats as programs make them, on the GPU: captured in a graph, with the cache's bytes compared; on two streams at a
time; on tensors that another stream made."""

import pytest
import torch

import mx4_ways
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def normal(shape, seed, dtype=BF):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def random_cache(n_pages, heads, page, dim, seed):
    cache = gs.mx4_cache(n_pages, heads, page, dim, DEV)
    table = torch.arange(n_pages, dtype=torch.int32, device=DEV).view(1, n_pages)
    k, v = (normal((1, n_pages * page, heads, dim), seed + i).to(DEV) for i in range(2))
    gs.mx4_cache_append(cache, table, torch.zeros(1, dtype=torch.int32, device=DEV), k, v)
    return cache


def test_a_captured_step_does_all_of_it():
    """Replays on a cache of their own: what they write and what they return is what an eager call writes and returns on another."""
    eager = random_cache(70, 2, 64, 64, 600)
    graphed = eager._replace(data=eager.data.clone())
    table = torch.randperm(70, generator=torch.Generator().manual_seed(601)).to(torch.int32).view(2, 35).to(DEV)
    w = gs.mx4_quantize(normal((256, 1003), 602).to(DEV))
    x = normal((40, 1003), 603).to(DEV)                                     # rows of odd length, padded first, shared sums
    lengths = torch.tensor([2100, 700], dtype=torch.int32, device=DEV)
    assert mx4_ways.dot_plan(True, 40, 256, 1003)[0].startswith("rows")
    big = gs.mx4_quantize(normal((100, 6203), 604).to(DEV))
    y = normal((17, 6203), 605).to(DEV)
    assert mx4_ways.dot_plan(True, 17, 100, 6203)[1] > 1

    def step(cache):
        a = gs.mx4_weight_dot(x, w, out_dtype=BF)[:2].contiguous()
        z = gs.mx4_dot(gs.mx4_quantize(a), gs.Mx4(w.values[:, :8].contiguous(), w.scales[:, :8].contiguous(), (256, 256), 1), out_dtype=BF)
        kv = z.view(2, 1, 4, 64)
        gs.mx4_cache_append(cache, table, lengths - 1, kv[:, :, :2].contiguous(), kv[:, :, 2:].contiguous())
        return gs.mx4_weight_dot(y, big), gs.mx4_attend(a.view(2, 1, 4, 64), cache, table, lengths, 0.125), z

    keep = eager.data.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed)
    graphed.data.copy_(keep)
    for i in range(4):
        x.copy_(normal((40, 1003), 610 + i))
        y.copy_(normal((17, 6203), 620 + i))
        lengths.add_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert not torch.equal(graphed.data, eager.data)                    # (the replay has written, the eager call not yet)
        want = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(graphed.data, eager.data)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_two_streams_at_a_time():
    """Products with shared sums and attention in parts on two streams, each with inputs and workspaces of its own: the results of calls alone."""
    jobs = []
    for i in range(2):
        cache = random_cache(70, 2, 64, 128, 700 + 10 * i)
        table = torch.randperm(70, generator=torch.Generator().manual_seed(701 + i)).to(torch.int32).view(1, 70).to(DEV)
        jobs.append((normal((17, 6203), 702 + i).to(DEV), gs.mx4_quantize(normal((100, 6203), 704 + i).to(DEV)), normal((1, 2, 8, 128), 706 + i).to(DEV),
                     cache, table, torch.tensor([4400 - 300 * i], dtype=torch.int32, device=DEV)))

    def work(job):
        x, w, q, cache, table, n = job
        return gs.mx4_weight_dot(x, w), gs.mx4_attend(q, cache, table, n, 0.09), gs.mx4_quantize(x).values

    alone = [work(job) for job in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(work(jobs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for results in got[i]:
            for a, b in zip(results, alone[i]):
                assert torch.equal(a, b)


def test_calls_go_to_the_current_stream():
    """On a stream that waits for the inputs' one, and back: a call on any other stream would not see them."""
    w = gs.mx4_quantize(normal((4096, 4096), 800).to(DEV))
    x = normal((300, 4096), 801).to(DEV)
    want = gs.mx4_weight_dot(x, w)
    torch.cuda.synchronize()
    for _ in range(5):
        side = torch.cuda.Stream()
        a = torch.zeros_like(x)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                a.copy_(x * 0.5)
            a.add_(a)
            got = gs.mx4_weight_dot(a, w)
            a.zero_()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        torch.cuda.synchronize()
