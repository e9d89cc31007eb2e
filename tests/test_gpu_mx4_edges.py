"""Operators on microscaled 4-bit floats at the ends of what their arguments may be, on the GPU.

Tolerances of attention as in test_gpu_mx4_ways.py: weights rounded to bfloat16 (2^-8 of the weighted sum of magnitudes and of the result), 2^-10 of that
sum for scores and exponentials, 2^-20 of the result for fp32 divisions and sums."""

import numpy as np
import pytest
import torch

import mx4_ways
from helpers import to_oracle
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, dtype=BF):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def cached(k, v, page):
    """A cache of one sequence that holds exactly these tokens (T, heads, dim), and its table."""
    tokens, heads, dim = k.shape
    width = -(-tokens // page)
    cache = gs.mx4_cache(width, heads, page, dim, DEV)
    table = torch.arange(width - 1, -1, -1, dtype=torch.int32).view(1, width)
    gs.mx4_cache_append(cache, table.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV), k[None].to(DEV), v[None].to(DEV))
    return cache, table


def check_attention(q, cache, table, length, scale):
    lens = torch.tensor([length], dtype=torch.int32)
    got = to_oracle(gs.mx4_attend(q.to(DEV), cache, table.to(DEV), lens.to(DEV), scale, out_dtype=F32))
    ref, mag = mx4_ways.attend(to_oracle(q), cache.data.cpu().numpy(), table.numpy(), lens.numpy(), cache.page_size, scale)
    tol = (2.0 ** -8 + 2.0 ** -10) * mag + (2.0 ** -8 + 2.0 ** -20) * np.abs(ref) + 1e-30
    err = np.abs(got - ref)
    assert np.isfinite(ref).all()
    worst = np.where(err <= tol, 0, err / tol).max()
    assert worst == 0, f"off by {worst} times what is allowed"


# queries and heads of a cache head, numbers per head: every attention kernel
KERNELS = [(1, 4, 64), (1, 3, 192), (2, 12, 128), (40, 1, 64), (10, 16, 128)]


@pytest.mark.parametrize("power", [20, 27, 29, 32, 40, 60, 100, 120])
@pytest.mark.parametrize("queries,group,dim", KERNELS)
def test_attention_with_far_scores(queries, group, dim, power):
    """Scores of 2^power, whose fp32 neighbours are many powers of e apart: the token with the largest one has all weight.  Keys are
    small whole numbers and each query is a power of two in one place, so that scores are exact, and no two largest are alike."""
    tokens = 150
    k = torch.randint(0, 4, (tokens, 1, dim), generator=torch.Generator().manual_seed(21)).float()
    at = torch.randint(0, 10, (dim,), generator=torch.Generator().manual_seed(22))
    k[at, 0, torch.arange(dim)] = 6.0            # one token per number, which the first query sees too: queries are the last of 150
    cache, table = cached(k, normal((tokens, 1, dim), 23, F32), 16)
    q = torch.zeros(1, queries, group, dim)
    place = torch.arange(queries * group).view(queries, group) * 5 % dim
    q[0, torch.arange(queries)[:, None], torch.arange(group)[None], place] = 2.0 ** power
    check_attention(q.to(BF), cache, table, tokens, 1.0)
    check_attention(-q.to(BF), cache, table, tokens, -1.0)
    check_attention((q * 2.0 ** -60).to(BF), cache, table, tokens, 2.0 ** 60)


@pytest.mark.parametrize("queries,group,dim", KERNELS)
def test_attention_with_far_scores_of_both_signs(queries, group, dim):
    """Rows whose scores are all far below zero, and rows near zero, in one wave."""
    tokens = 150
    k, v = normal((tokens, 1, dim), 31, F32), normal((tokens, 1, dim), 32, F32)
    k[:, :, 0] = torch.arange(tokens).float()[:, None] % 3 + 2.0
    cache, table = cached(k, v, 16)
    q = 0.1 * normal((1, queries, group, dim), 33, F32)
    far = (torch.arange(queries)[:, None] + torch.arange(group)[None]) % 2 == 0
    q[0, far] = 0.0
    q[0, far, 0] = -2.0 ** 33                    # the mean over a third of the tokens
    check_attention(q.to(BF), cache, table, tokens, 1.0)


@pytest.mark.parametrize("scale", [2.0 ** 127, -2.0 ** 127, 2.358e38])
@pytest.mark.parametrize("queries,group,dim", KERNELS)
def test_attention_with_the_largest_scales(queries, group, dim, scale):
    """Up to those that are refused: scores of zero, scores of some units, and scores so far apart that one token has all weight."""
    tokens = 70
    k, v = normal((tokens, 1, dim), 11, F32), normal((tokens, 1, dim), 12, F32)
    cache, table = cached(k, v, 16)
    q = normal((1, queries, group, dim), 13, F32)
    tiny = q * 2.0 ** -128                       # numbers below bfloat16's normal ones, scores of some units
    tiny[:, :, 0] = 0.0                          # the mean of the values
    check_attention(tiny.to(BF), cache, table, tokens, scale)
    check_attention((q * 2.0 ** -60).to(BF), cache, table, tokens, scale)


@pytest.mark.parametrize("scale", [2.0 ** -125, 1e-39, -1e-39, 2.0 ** -134])
@pytest.mark.parametrize("queries,group,dim", KERNELS)
def test_attention_with_the_smallest_scales(queries, group, dim, scale):
    """Scales beyond float's normal numbers, and queries so large that scores are some units all the same (2^-134 has 16 bits left: off by 2^-17 of scores
    below 8)."""
    tokens = 60
    k, v = normal((tokens, 1, dim), 41, F32), normal((tokens, 1, dim), 42, F32)
    cache, table = cached(0.25 * k, v, 16)
    q = normal((1, queries, group, dim), 43, F32) * 2.0 ** 122
    check_attention(q.to(BF), cache, table, tokens, scale)


@pytest.mark.parametrize("queries", [1, 40])
def test_a_cache_without_pages(queries):
    """Tokens are dropped, read back as zeros, and seen by nobody."""
    cache = gs.mx4_cache(0, 2, 16, 64, DEV)
    table = torch.zeros(3, 5, dtype=torch.int32, device=DEV)
    n = torch.tensor([80, 0, 7], dtype=torch.int32, device=DEV)
    k = normal((3, 9, 2, 64), 51).to(DEV)
    gs.mx4_cache_append(cache, table, n, k, k)
    for got in gs.mx4_cache_read(cache, table, n, 9):
        assert got.shape == k.shape and not got.any()
    assert not gs.mx4_attend(normal((3, queries, 4, 64), 52).to(DEV), cache, table, n, 0.1).any()


@pytest.mark.parametrize("power,tolerance", [(-100, 2.0 ** -20), (-112, 2.0 ** -8), (-124, 2.0 ** 4)])
@pytest.mark.parametrize("queries,group,dim", KERNELS)
def test_attention_over_the_smallest_values(queries, group, dim, power, tolerance):
    """Weights are 2^-24 times as large until they are divided by their sum, and a product with a value has the bits down to 2^-149: each of 60
    is off by 2^-150 at most, 2^-126 in the result, 60 of them by less than 2^-120 in all; `tolerance` is that over the values' size."""
    tokens = 60
    k, v = normal((tokens, 1, dim), 61, F32), normal((tokens, 1, dim), 62, F32) * 2.0 ** power
    cache, table = cached(k, v, 16)
    lens = torch.tensor([tokens], dtype=torch.int32)
    q = normal((1, queries, group, dim), 63)
    got = to_oracle(gs.mx4_attend(q.to(DEV), cache, table.to(DEV), lens.to(DEV), dim ** -0.5, out_dtype=F32))
    ref, mag = mx4_ways.attend(to_oracle(q), cache.data.cpu().numpy(), table.numpy(), lens.numpy(), 16, dim ** -0.5)
    tol = (2.0 ** -8 + 2.0 ** -10) * mag + (2.0 ** -8 + 2.0 ** -20) * np.abs(ref) + tolerance * 2.0 ** power
    assert (np.abs(got - ref) <= tol).all()
