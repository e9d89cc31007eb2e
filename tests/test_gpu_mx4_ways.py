"""Products and attention on microscaled 4-bit floats in every way that the library has (mx4_ways.py), on the GPU against float64.

Tolerances from the arithmetic.  Products: those of two numbers are exact in fp32, their sums over K off by at most K 2^-24 of the
sum of magnitudes, a bfloat16 result by 2^-8 of its value more.  Attention: weights are rounded to bfloat16, those under the line too, so that
a result is off by 2^-8 of the weighted sum of magnitudes and of itself; fp32 scores and their exponentials add at most 2^-10 of
that sum for scores below 64; then the result's own rounding."""

import numpy as np
import pytest
import torch

import mx4_ways
from helpers import to_oracle
from oracle import mx4
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, dtype=BF):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def scattered_cache(case, seed):
    """Tokens of all sequences in scattered pages, a little of everything that may be there beside them: entries that are no page,
    value scales of 2^126 and more and NaN, all ones behind the last token."""
    batch, heads, dim, page = (case[k] for k in ("batch", "heads", "dim", "page"))
    width = -(-case["longest"] // page)
    n_pages = batch * width + 2
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:batch * width].view(batch, width).to(torch.int32)
    cache = gs.mx4_cache(n_pages, heads, page, dim, DEV)
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)
    k, v = (0.5 * torch.randn((batch, width * page, heads, dim), generator=gen, device=DEV) for _ in range(2))
    gs.mx4_cache_append(cache, table.to(DEV), torch.zeros(batch, dtype=torch.int32, device=DEV), k, v)
    data = cache.data.cpu()
    lens = mx4_ways.lengths(case)
    blocks, first = dim // 32, lens[0]
    for token, block, byte, head in ((first - 3, 0, 253, slice(None)), (first - 20, blocks - 1, 255, 0), (first - 90, 0, 254, heads - 1)):
        data[int(table[0, token // page]), head, int(mx4.token_offsets(page, dim, token % page)[3][block])] = byte
    for b in range(batch):
        for token in range(lens[b], min(-(-lens[b] // page) * page, lens[b] + 70)):
            for part in mx4.token_offsets(page, dim, token % page):
                data[int(table[b, token // page]), :, part] = 255
    if width > 2:
        table[-1, width // 2], table[-1, 1] = -1, 10 ** 6
    cache.data.copy_(data)
    return cache, table, torch.tensor(lens, dtype=torch.int32)


@pytest.mark.parametrize("case", mx4_ways.ATTENTIONS, ids=lambda c: "{way}-{dim}".format(**c))
def test_attention(case):
    seed = 1000 + case["dim"] + 10 * case["longest"] + case["batch"]
    cache, table, lens = scattered_cache(case, seed)
    q = normal((case["batch"], case["queries"], case["heads"] * case["group"], case["dim"]), seed + 2)
    scale = case["dim"] ** -0.5
    data, rows = cache.data.cpu().numpy(), to_oracle(q)
    for (window, sinks), odt in zip(mx4_ways.windows(case), (F32, BF)):
        assert mx4_ways.attend_plan(case, window, sinks) == case["way"]
        ref, mag = mx4_ways.attend(rows, data, table.numpy(), lens.numpy(), case["page"], scale, window, sinks)
        out = torch.full(q.shape, 9.0, dtype=odt, device=DEV)
        gs.mx4_attend(q.to(DEV), cache, table.to(DEV), lens.to(DEV), scale, window=window, sinks=sinks, out=out,
                      workspace=torch.full((1 << 26,), 255, dtype=torch.uint8, device=DEV))      # (NaN: nothing unwritten is read)
        got, nan = to_oracle(out), np.isnan(ref)
        assert nan.any() and np.array_equal(np.isnan(got), nan)
        ref, got, mag = (np.where(nan, 0, x) for x in (ref, got, mag))
        tol = (2.0 ** -8 + 2.0 ** -10) * mag + (2.0 ** -8 + (2.0 ** -8 if odt == BF else 2.0 ** -20)) * np.abs(ref) + 1e-30
        err = np.abs(got - ref)
        assert (err <= tol).all(), f"window {window}: off by {(err / tol).max()} times what is allowed"


def check_product(got, x, w):
    ref, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    tol = x.shape[1] * 2.0 ** -24 * mag + (2.0 ** -8 * np.abs(ref) if got.dtype == BF else 0)
    err = np.abs(to_oracle(got) - ref)
    assert (err <= tol).all(), f"off by {(err - tol).max()} more than allowed"


def stored(m):
    rows, k = m.shape
    return mx4.dequantize(m.values.cpu().numpy().reshape(rows, -1, 16), m.scales.cpu().numpy().reshape(rows, -1), k)


@pytest.mark.parametrize("key", mx4_ways.DOTS, ids=str)
def test_dot(key):
    m, n, k = mx4_ways.DOTS[key]
    assert mx4_ways.dot_plan(False, m, n, k) == (key[0], 1)
    x, w = (gs.mx4_quantize(normal(shape, 2000 + k + i).to(DEV)) for i, shape in enumerate(((m, k), (n, k))))
    check_product(gs.mx4_dot(x, w, out_dtype=BF if k % 3 else F32), stored(x), stored(w))


@pytest.mark.parametrize("key", mx4_ways.WEIGHT_DOTS, ids=str)
def test_weight_dot(key):
    m, n, k = mx4_ways.WEIGHT_DOTS[key]
    way, splits = mx4_ways.dot_plan(True, m, n, k)
    assert (way, splits > 1) == key[:2]
    x, w = normal((m, k), 3000 + k), gs.mx4_quantize(normal((n, k), 3001 + k).to(DEV))
    check_product(gs.mx4_weight_dot(x.to(DEV), w, out_dtype=F32 if k % 3 else BF), to_oracle(x), stored(w))
