"""The stack of 4-bit decoder layers on the GPU against the same sequence in float64 with the oracle's conversions.

Each call is checked by itself elsewhere; here it is that they fit together.  Every result of a call is rounded to bfloat16 on both sides.
What a call computes is off by a rounding of its result (2^-8, relative), the attention by 2^-8 of the weights more; a quantised number
next to a border between two codes may fall on the other side, a quarter of its magnitude.  A bound from these would be far above what
happens, so agreement is measured in the 2-norm: a rounding of every element by the largest amount in each of a layer's 9 calls, all in
the same direction, is 9 * 2^-8 = 3.5 % per layer; conversions that fall on the other side are as rare as values within 2^-8 of one of the borders
(a few in 100) and each moves its block by 1/4 at most: another 5 % of the norm of what they go into at the most.
"""

import numpy as np
import pytest
import torch

from helpers import to_oracle
from oracle import mx4
from paper_2105_09377_amd import binding as gs
from paper_2105_09377_amd import decoder4, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WIDTH, HEADS, KV, DIM, HIDDEN = 320, 8, 2, 64, 700


def layers(n):
    out = []
    for i in range(n):
        shapes = decoder4.weight_shapes(WIDTH, HEADS, KV, DIM, HIDDEN)
        out.append({name: synth.normal_bf16(shape, 0.5 * shape[1] ** -0.5, 9000 + 10 * i + j) for j, (name, shape) in enumerate(shapes.items())})
    return out


def stack(n, **kw):
    return decoder4.Decoder4Stack(layers(n), HEADS, KV, DIM, n_pages=24, page_size=16, device=DEV, **kw)


def bf(x):
    return to_oracle(torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16))


def small(x):
    flat = x.reshape(-1, x.shape[-1])
    return mx4.dequantize(*mx4.quantize(flat), x.shape[-1]).reshape(x.shape)


def reference(ws, x, window, sinks, quantize):
    """All tokens x (T, width) of one sequence at once, no cache: a token attends to the quantised keys in front of it."""
    n = x.shape[0]
    for w in ws:
        w = {name: small(to_oracle(t)) for name, t in w.items()}
        q, k, v = (bf(x @ w[name].T).reshape(n, -1, DIM) for name in "qkv")
        k, v = np.repeat(small(k), HEADS // KV, 1), np.repeat(small(v), HEADS // KV, 1)
        s = np.einsum("ihd,thd->hit", q, k) * DIM ** -0.5
        ago = np.arange(n)[:, None] - np.arange(n)[None]
        hidden = (ago < 0) | ((ago >= window) & (np.arange(n)[None] >= sinks) if window else False)
        s = np.where(hidden, -np.inf, s)
        p = np.exp(s - s.max(-1, keepdims=True))
        a = bf(np.einsum("hit,thd->ihd", p / p.sum(-1, keepdims=True), v).reshape(n, -1))
        x = bf(x + bf(a @ w["o"].T))
        h = bf(np.maximum((small(x) if quantize else x) @ w["up"].T, 0))
        x = bf(x + bf((small(h) if quantize else h) @ w["down"].T))
    return x


def run(st, x, pieces, table):
    """Two sequences fed in pieces of so many tokens, the second one a token behind the first."""
    out, at = [], 0
    for n in pieces:
        first = torch.full((2,), at, dtype=torch.int32, device=DEV)
        out.append(st.step(x[:, at:at + n].contiguous(), table, first, first + n))
        at += n
    return torch.cat(out, 1)


@pytest.mark.parametrize("window,sinks,quantize", [(0, 0, False), (20, 3, False), (0, 0, True)])
@pytest.mark.parametrize("pieces", [(70,), (1,) * 6 + (40, 23, 1), (33, 37)])
def test_against_the_definition(pieces, window, sinks, quantize):
    ws = layers(2)
    st = stack(2, window=window, sinks=sinks, quantize_rows=0 if quantize else None)
    x = synth.normal_bf16((2, 70, WIDTH), 1.0, 9100)
    table = torch.randperm(24, generator=torch.Generator().manual_seed(1))[:10].view(2, 5).to(torch.int32).to(DEV)
    got = run(st, x.to(DEV), pieces, table)
    for b in range(2):
        want = reference(ws, to_oracle(x[b]), window, sinks, quantize)
        off = np.linalg.norm(to_oracle(got[b]) - want) / np.linalg.norm(want)
        assert off <= 2 * (9 * 2.0 ** -8 + (0.05 if quantize else 0.02)), off


def test_a_captured_token_equals_an_eager_one():
    table = torch.arange(20, dtype=torch.int32, device=DEV).view(2, 10)
    eager, graphed = stack(2), stack(2)
    x = synth.normal_bf16((2, 40, WIDTH), 1.0, 9200).to(DEV)
    first = torch.zeros(2, dtype=torch.int32, device=DEV)
    for st in (eager, graphed):
        st.step(x[:, :30].contiguous(), table, first, first + 30)
    token, at, n = x[:, 30:31].clone(), first + 30, first + 31
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(token, table, at, n)                # (writes what the first replay writes again)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = graphed.step(token, table, at, n)
    for i in range(30, 36):
        token.copy_(x[:, i:i + 1])
        at.fill_(i)
        n.fill_(i + 1)
        want = eager.step(token, table, at, n)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
