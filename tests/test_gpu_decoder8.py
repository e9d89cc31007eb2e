"""The stack of 8-bit decoder layers with experts on the GPU against its definition in float64 (decoder8_reference.py, which says what is
allowed; mistakes planted in it are beyond that, test_decoder8_host.py)."""

import pytest
import torch

import decoder8_reference as ref
from helpers import to_oracle
from paper_2105_09377_amd import binding as gs
from paper_2105_09377_amd import decoder8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BATCH = 2


class Routes:
    """The reference's routing for the tokens from `at` on, as many as a step has; counts of what it was asked."""

    def __init__(self):
        self.at, self.seen = 0, []
        self.tables = {i: tuple(t.to(DEV) for t in ref.routing(i, BATCH)) for i in range(2)}

    def __call__(self, layer, y):
        n = y.shape[0] // BATCH
        self.seen.append((layer, y.shape, y.n_access, y.block_rows))
        return tuple(t[:, self.at:self.at + n].reshape(BATCH * n, ref.CHOICES).contiguous() for t in self.tables[layer])


def stack(n, routes):
    return decoder8.Decoder8Stack(ref.layers(n), ref.HEADS, ref.KV, ref.DIM, n_pages=24, page_size=16, route=routes, eps=1e-5, device=DEV)


def run(st, routes, x, pieces, table):
    out = []
    for n in pieces:
        at = routes.at
        first = torch.full((BATCH,), at, dtype=torch.int32, device=DEV)
        out.append(st.step(x[:, at:at + n].contiguous(), table, first, first + n))
        routes.at += n
    return torch.cat(out, 1)


TABLE = torch.randperm(24, generator=torch.Generator().manual_seed(1))[:10].view(2, 5).to(torch.int32)


@pytest.mark.parametrize("pieces", [(ref.TOKENS,), ref.PIECES])
@pytest.mark.parametrize("n", [1, 2])
def test_against_the_definition(n, pieces):
    routes = Routes()
    x = ref.tokens(BATCH)
    got = run(stack(n, routes), routes, x.to(DEV), pieces, TABLE.to(DEV))
    assert routes.seen[0] == (0, (BATCH * pieces[0], ref.WIDTH), 1, 1) and len(routes.seen) == n * len(pieces)
    for b in range(BATCH):
        xv = to_oracle(x[b])
        want = ref.stack(n, xv, b, BATCH)
        off, limit = ref.off(to_oracle(got[b]), want, xv), ref.allowed(xv, n, b, BATCH)
        assert off <= limit, (off, limit)


def test_pieces_do_not_matter():
    """A token's result has the same bits whether it comes alone or with the tokens in front of it, where its products are done in the same way."""
    whole, parts = Routes(), Routes()
    x = ref.tokens(BATCH).to(DEV)[:, :6].contiguous()
    a = run(stack(2, whole), whole, x, (6,), TABLE.to(DEV))
    b = run(stack(2, parts), parts, x, (1, 2, 3), TABLE.to(DEV))
    assert ref.off(to_oracle(b), to_oracle(a), to_oracle(x)) <= 0.02


def test_a_captured_token_equals_an_eager_one():
    routes = {"eager": Routes(), "graphed": Routes()}
    stacks = {name: stack(2, r) for name, r in routes.items()}
    x, table = ref.tokens(BATCH).to(DEV), TABLE.to(DEV)
    for name in stacks:
        run(stacks[name], routes[name], x, (30,), table)
    token, at, n = x[:, 30:31].clone(), torch.full((BATCH,), 30, dtype=torch.int32, device=DEV), torch.full((BATCH,), 31, dtype=torch.int32, device=DEV)
    # the graph's experts are read from tensors of its own
    held = {i: tuple(t[:, 30].clone() for t in routes["graphed"].tables[i]) for i in range(2)}
    stacks["graphed"].route = lambda layer, y: held[layer]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stacks["graphed"].step(token, table, at, n)                # (writes what the first replay writes again)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = stacks["graphed"].step(token, table, at, n)
    for i in range(30, 36):
        token.copy_(x[:, i:i + 1])
        at.fill_(i)
        n.fill_(i + 1)
        for layer in range(2):
            for mine, all_of in zip(held[layer], routes["eager"].tables[layer]):
                mine.copy_(all_of[:, i])
        routes["eager"].at = i
        want = stacks["eager"].step(token, table, at, n)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_no_layers_and_no_tokens():
    st = decoder8.Decoder8Stack([], ref.HEADS, ref.KV, ref.DIM, n_pages=1, page_size=16, route=None, device=DEV)
    x = ref.tokens(BATCH).to(DEV)
    assert torch.equal(st.step(x, TABLE.to(DEV), None, None), x)
    routes = Routes()
    none = torch.zeros(BATCH, dtype=torch.int32, device=DEV)
    assert stack(1, routes).step(x[:, :0].contiguous(), TABLE.to(DEV), none, none).shape == (BATCH, 0, ref.WIDTH)
