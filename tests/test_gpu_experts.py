"""Tokens dealt to experts on the GPU against the oracle in float64.

Sorting and spreading out are compared exactly.  Tolerances of the rest, from the arithmetic: sums of c products in fp32 are off by at
most (c + 1) 2^-24 of the sum of their magnitudes, a result by half a step of its type more; products of the experts as those of
test_gpu_f8.py.
"""

import numpy as np
import pytest
import torch

from helpers import to_oracle
from oracle import f8
from paper_2105_09377_amd import binding as gs
from test_gpu_f8 import BF, DEV, EPS, F32, allowed, normal, operand, within

pytestmark = pytest.mark.gpu
I32 = torch.int32


def chosen(tokens, choices, experts, seed, dropped=0.1):
    """Experts of every token, some of them none (below zero and above), the same one twice now and then."""
    g = torch.Generator().manual_seed(seed)
    e = torch.randint(0, max(experts, 1), (tokens, choices), generator=g)
    e = torch.where(torch.rand(tokens, choices, generator=g) < 0.3, e // 3, e)
    odd = torch.tensor([-1, experts, 2 ** 31 - 1, -2 ** 31])[torch.randint(0, 4, (tokens, choices), generator=g)]
    return torch.where(torch.rand(tokens, choices, generator=g) < dropped, odd, e).to(I32)


def same(got, want):
    assert got.dtype == I32 and np.array_equal(to_oracle(got), want)


# ------------------------------------------------------------------------------------------------
# sorting
# ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("tokens,choices,experts", [(1, 1, 1), (1, 8, 8), (5, 2, 3), (64, 1, 64), (65, 2, 1), (33, 4, 60), (200, 6, 257), (1000, 2, 16),
                                                    (1500, 2, 4096), (4097, 1, 5), (3000, 3, 128), (5000, 8, 64), (20000, 2, 300), (70001, 1, 2000)])
def test_sort(tokens, choices, experts):
    e = chosen(tokens, choices, experts, tokens + experts)
    s = gs.expert_sort(e.to(DEV), experts)
    for got, want in zip(s, f8.sort(e.numpy(), experts)):
        same(got, want)


@pytest.mark.parametrize("tokens", [0, 7, 9000])
def test_sort_nothing(tokens):
    s = gs.expert_sort(torch.full((tokens, 2), -1, dtype=I32, device=DEV), 5)
    assert not s.offsets.any() and (s.tokens == -1).all() and (s.places == -1).all() and s.tokens.numel() == 2 * tokens
    s = gs.expert_sort(torch.zeros((tokens, 2), dtype=I32, device=DEV), 0)
    assert s.offsets.tolist() == [0] and (s.places == -1).all()
    assert gs.expert_sort(torch.zeros((tokens, 0), dtype=I32, device=DEV), 4).offsets.tolist() == [0] * 5


def test_sort_one_expert_has_all():
    for tokens in (100, 10000):
        s = gs.expert_sort(torch.full((tokens, 2), 3, dtype=I32, device=DEV), 5)
        assert s.offsets.tolist() == [0, 0, 0, 0, 2 * tokens, 2 * tokens]
        assert torch.equal(s.places.flatten().cpu(), torch.arange(2 * tokens, dtype=I32))


# ------------------------------------------------------------------------------------------------
# rows
# ------------------------------------------------------------------------------------------------

ROWS = [(1, 1, 1, 1), (1, 8, 8, 7), (5, 2, 3, 8), (33, 4, 60, 100), (100, 6, 16, 257), (64, 3, 8, 1024), (300, 5, 16, 2050), (3000, 2, 16, 64)]


@pytest.mark.parametrize("dtype", [BF, F32, torch.int8, I32, torch.float8_e4m3fn])
@pytest.mark.parametrize("tokens,choices,experts,cols", ROWS)
def test_split(tokens, choices, experts, cols, dtype):
    e = chosen(tokens, choices, experts, cols)
    s = gs.expert_sort(e.to(DEV), experts)
    x = (normal((tokens, cols), 1, F32) * 20).to(dtype)
    rows = torch.full((tokens * choices, cols), 5, dtype=F32).to(dtype)
    got = gs.expert_split(x.to(DEV), s.places, out=rows.to(DEV))
    assert np.array_equal(to_oracle(got), f8.split(to_oracle(x), f8.sort(e.numpy(), experts)[2], to_oracle(rows)))


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,choices,experts,cols", ROWS)
def test_join_and_its_gradient(tokens, choices, experts, cols, dtype, weighted):
    e = chosen(tokens, choices, experts, cols)
    s = gs.expert_sort(e.to(DEV), experts)
    places = f8.sort(e.numpy(), experts)[2]
    rows, grad = normal((tokens * choices, cols), 2, dtype), normal((tokens, cols), 3, dtype)
    weights = normal((tokens, choices), 4, F32) if weighted else None
    on, wv = (weights.to(DEV), to_oracle(weights)) if weighted else (None, None)
    for odt in (BF, F32):
        want, size = f8.join(to_oracle(rows), places, wv)
        got = gs.expert_join(rows.to(DEV), s.places, on, out_dtype=odt)
        assert got.dtype == odt
        slack = size * (choices + 1) * 2.0 ** -24
        within(got, want, slack + (np.abs(want) + slack) * EPS[odt])
    before = normal((tokens * choices, cols), 9, dtype)
    got_rows, got_weights = gs.expert_join_grad(grad.to(DEV), rows.to(DEV), s.places, on, grad_rows=before.to(DEV))
    want_rows, want_weights, size = f8.join_grad(to_oracle(grad), to_oracle(rows), places, wv, to_oracle(before))
    within(got_rows, want_rows, np.abs(want_rows) * (EPS[dtype] + 2.0 ** -24) * (1 + 2.0 ** -7))
    within(got_weights, want_weights, size * (cols + 1) * 2.0 ** -24)
    held = s.places.flatten().long()
    free = torch.ones(tokens * choices, dtype=torch.bool)
    free[held[held >= 0].cpu()] = False
    assert torch.equal(got_rows.cpu()[free], before[free])


def test_gradients_are_differences():
    """Of sum(grad * join(split(x), weights)) in x, the rows and the weights: it is linear in each, so that differences are exact up to
    rounding, 2^-22 of the sum of magnitudes."""
    tokens, choices, cols = 13, 3, 40
    e = chosen(tokens, choices, 6, 1)
    s = gs.expert_sort(e.to(DEV), 6)
    x, grad, weights = normal((tokens, cols), 1, F32).to(DEV), normal((tokens, cols), 2, F32).to(DEV), normal((tokens, choices), 3, F32).to(DEV)
    rows = gs.expert_split(x, s.places, out=torch.zeros(tokens * choices, cols, device=DEV))
    grad_rows, grad_weights = gs.expert_join_grad(grad, rows, s.places, weights, grad_rows=torch.zeros_like(rows))
    grad_x = gs.expert_join(grad_rows, s.places)

    def loss(x, rows, weights):
        rows = gs.expert_split(x, s.places, out=torch.zeros(tokens * choices, cols, device=DEV)) if rows is None else rows
        y = gs.expert_join(rows, s.places, weights).double() * grad.double()
        return y.sum().item(), y.abs().sum().item()

    base, size = loss(x, None, weights)
    for what, of, by in (("x", x, grad_x), ("rows", rows, grad_rows), ("weights", weights, grad_weights)):
        step = normal(tuple(of.shape), 7, F32).to(DEV)
        moved = (of + step)
        step = moved.double() - of.double()
        args = {"x": (moved, None, weights), "rows": (x, moved, weights), "weights": (x, None, moved)}[what]
        value, more = loss(*args)
        terms = (step.abs() * by.abs().double()).sum().item()
        assert abs((value - base) - (step * by.double()).sum().item()) <= (size + more + terms) * (choices + cols + 4) * 2.0 ** -24, what


def test_rows_of_any_place():
    """Places that are no rows, of a table that nobody sorted; fewer rows than choices."""
    places = torch.tensor([[3, -1], [4, 0], [-7, 2 ** 31 - 1], [1, 2]], dtype=I32)
    x, rows = normal((4, 37), 1), normal((4, 37), 2)
    got = gs.expert_split(x.to(DEV), places.to(DEV), out=rows.to(DEV))
    assert np.array_equal(to_oracle(got), f8.split(to_oracle(x), places.numpy(), to_oracle(rows)))
    weights = torch.tensor([[1.0, float("nan")], [float("inf"), 2.0], [float("nan"), float("nan")], [-1.0, 0.5]])
    want, size = f8.join(to_oracle(rows), places.numpy(), np.nan_to_num(to_oracle(weights), posinf=0.0))
    within(gs.expert_join(rows.to(DEV), places.to(DEV), weights.to(DEV)), want, size * 2.0 ** -20 + np.abs(want) * 2.0 ** -7)


def test_rows_of_several_dimensions():
    x, places = normal((4, 3, 5), 1, F32).to(DEV), torch.tensor([[0], [1], [2], [3]], dtype=I32, device=DEV)
    rows = gs.expert_split(x, places)
    assert torch.equal(rows, x) and torch.equal(gs.expert_join(rows, places), x)


def test_no_choices():
    x, places = normal((4, 8), 1, F32).to(DEV), torch.zeros((4, 0), dtype=I32, device=DEV)
    assert gs.expert_split(x, places).shape == (0, 8)
    assert not gs.expert_join(torch.zeros((0, 8), device=DEV), places, out=torch.ones(4, 8, device=DEV)).any()
    a, b = gs.expert_join_grad(x, torch.zeros((0, 8), device=DEV), places)
    assert a.shape == (0, 8) and b.shape == (4, 0)


# ------------------------------------------------------------------------------------------------
# the experts' products
# ------------------------------------------------------------------------------------------------


def check_experts(tokens, choices, experts, n, k, gather, w_rows=128, odt=BF, act=gs.GS_ACT_NONE, dropped=0.1, e=None, x_rows=1):
    e = chosen(tokens, choices, experts, n + k, dropped) if e is None else e
    offsets, of, _ = f8.sort(e.numpy(), experts)
    rows = e.numel()
    x, xv = operand((tokens if gather else rows, k), 1, x_rows, 1)
    w, wv = operand((experts, n, k), 2, w_rows, 2)
    before = normal((rows, n), 3, odt)
    got = gs.f8_expert_dot(x, w, torch.from_numpy(offsets).to(I32).to(DEV), tokens=torch.from_numpy(of).to(I32).to(DEV) if gather else None,
                           act=act, out=before.to(DEV))
    want, size = f8.expert_dot(xv[0], of if gather else None, offsets, wv, np.zeros((rows, n)))
    if act == gs.GS_ACT_RELU:
        want = np.maximum(want, 0)
    last = int(offsets[-1])
    within(got[:last], want[:last], allowed(size[:last], want[:last], -(-k // 128), odt))
    assert torch.equal(got[last:].cpu(), before[last:])


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("tokens,choices,experts,n,k", [(1, 1, 1, 1, 1), (1, 2, 8, 130, 300), (4, 2, 3, 64, 128), (20, 4, 60, 200, 513), (3, 8, 70, 33, 1030),
                                                        (100, 2, 4, 256, 384), (500, 2, 3, 300, 260), (700, 1, 16, 513, 130), (1500, 2, 5, 520, 390)])
def test_expert_dot(tokens, choices, experts, n, k, gather):
    check_experts(tokens, choices, experts, n, k, gather)


@pytest.mark.parametrize("tokens", [6, 900])
def test_expert_dot_kinds(tokens):
    check_experts(tokens, 2, 4, 300, 200, True, w_rows=1, odt=F32)
    check_experts(tokens, 2, 4, 300, 200, False, act=gs.GS_ACT_RELU)
    check_experts(tokens, 2, 4, 140, 700, True, x_rows=128)
    check_experts(tokens, 2, 4, 140, 700, False, x_rows=128, w_rows=1)


@pytest.mark.parametrize("tokens", [9, 700])
def test_expert_dot_uneven(tokens):
    """One expert has all rows; most have none; all choices dropped."""
    for e in (3, 0, 65, -1):
        check_experts(tokens, 2, 66, 140, 200, True, e=torch.full((tokens, 2), e, dtype=I32))


@pytest.mark.parametrize("rows", [12, 600])
def test_expert_dot_any_offsets(rows):
    """Tables that nobody sorted: tokens that are none, offsets beyond the rows or in no order; every access stays in bounds and rows of
    no expert as they were."""
    n, k = 140, 200
    (x, xv), (w, wv) = operand((7, k), 1, 1, 1), operand((4, n, k), 2, 128, 2)
    tokens = torch.arange(rows) % 10 - 2
    for offsets in ([0, 3, 3, rows // 2, rows], [-5, 2, 5, 6, rows + 100], [4, 5, 5, 6, 7], [0, 0, 0, 0, 0]):
        before = normal((rows, n), 3, F32)
        got = gs.f8_expert_dot(x, w, torch.tensor(offsets, dtype=I32, device=DEV), tokens=tokens.to(I32).to(DEV), out=before.to(DEV))
        want, size = f8.expert_dot(xv[0], tokens.numpy(), offsets, wv, to_oracle(before))
        within(got, want, np.where(size > 0, allowed(size, want, 2, F32), 0))
    offsets = torch.tensor([rows, 2 ** 31 - 1, -2 ** 31, 3, 1], dtype=I32, device=DEV)
    gs.f8_expert_dot(x, w, offsets, tokens=tokens.to(I32).to(DEV))
    torch.cuda.synchronize()


def test_expert_dot_nan_stays_in_its_row():
    k, n = 200, 70
    x = normal((6, k), 1, F32)
    x[2, 3] = float("nan")
    xq, (w, _) = gs.f8_quantize(x.to(DEV)), operand((2, n, k), 2, 128, 2)
    for rows in (8, 400):
        tokens = torch.arange(rows) % 7 - 1
        got = gs.f8_expert_dot(xq, w, torch.tensor([0, rows // 2, rows], dtype=I32, device=DEV), tokens=tokens.to(I32).to(DEV)).cpu()
        assert torch.equal(torch.isnan(got).all(1), tokens == 2) and torch.equal(torch.isnan(got).any(1), tokens == 2)
        assert (got[tokens < 0] == 0).all()


def test_no_experts():
    x, out = operand((64, 200), 1, 1, 1)[0], torch.ones(64, 70, device=DEV)
    w = gs.F8(torch.zeros(0, 70, 2, 128, dtype=torch.uint8, device=DEV), torch.zeros(0, 1, 4, device=DEV), (0, 70, 200), 2, 128)
    gs.f8_expert_dot(x, w, torch.zeros(1, dtype=I32, device=DEV), out=out)
    assert (out == 1).all()


def test_no_rows_and_no_tokens():
    w = operand((2, 70, 200), 2, 128, 2)[0]
    none = gs.f8_quantize(torch.zeros(0, 200, device=DEV))
    out = gs.f8_expert_dot(none, w, torch.zeros(3, dtype=I32, device=DEV))
    assert out.shape == (0, 70)
    out = torch.ones(5, 70, device=DEV)
    gs.f8_expert_dot(none, w, torch.tensor([0, 2, 4], dtype=I32, device=DEV), tokens=torch.zeros(5, dtype=I32, device=DEV), out=out)
    assert not out[:4].any() and (out[4] == 1).all()
