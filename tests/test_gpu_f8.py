"""Scaled 8-bit floats and norms on the GPU against the oracle in float64.

Quantising is compared bit for bit.  Tolerances of the rest, from the arithmetic:
* products: the matrix unit adds the products of a block aligned to the largest (2^-13 of the sum of their magnitudes, see
  helpers.fp8_slack); the block's sum times the product of two scales, itself rounded, is added to the result: 2 roundings of each term and
  as many of the running sum as there are blocks, each at most 2^-24 of the sum of all magnitudes; the result's own rounding;
* norms: 64 bits until they are rounded to float: half a step of it and a few of 2^-52, then the result's own rounding; their codes are those
  of the float nearest to the norm, bit for bit (a norm that is within 2^-50 of the middle between two floats may have the other
  neighbour: that is 1 in 2^26).
"""

import numpy as np
import pytest
import torch

from helpers import to_oracle
from oracle import f8
from paper_2105_09377_amd import binding as gs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
EPS = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def normal(shape, seed, dtype=BF, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if spread:
        x = x * torch.exp2(torch.randn(shape[:-1] + (1,), generator=g) * spread)
    return x.to(dtype)


def codes_of(m):
    return m.values.view(torch.uint8).cpu().numpy()


def same_scales(got, want):
    got = to_oracle(got)
    assert got.shape == want.shape and np.array_equal(got, want, equal_nan=True)


def within(got, want, allowed):
    got = to_oracle(got)
    assert got.shape == want.shape
    off = np.abs(got - want) - allowed
    assert not np.isnan(off).any() and (off <= 0).all(), f"off by {off.max()} more than allowed"


# ------------------------------------------------------------------------------------------------
# conversions
# ------------------------------------------------------------------------------------------------

SHAPES = [(1, 1), (1, 127), (3, 128), (5, 129), (2, 511), (7, 512), (4, 513), (1, 4096), (129, 1000), (64, 2047), (1000, 7), (300, 130)]


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize(rows, cols, dtype, block_rows):
    x = normal((rows, cols), 100 + rows + cols, dtype, spread=6.0)
    x[0, 0] = 0.0
    if rows > 2:
        x[1] = 0.0
        x[2, cols // 2] = -0.0
    m = gs.f8_quantize(x.to(DEV), block_rows=block_rows)
    code, scales = f8.quantize(to_oracle(x)[None], block_rows)
    assert m.shape == (rows, cols) and m.n_access == 1 and m.block_rows == block_rows
    assert np.array_equal(codes_of(m), code[0])
    same_scales(m.scales, scales[0])
    want = f8.dequantize(code, scales, cols, block_rows)[0]
    for odt in (BF, F32):
        got = gs.f8_dequantize(m, out_dtype=odt)
        assert got.dtype == odt and got.shape == (rows, cols)
        once = torch.from_numpy(f8.round32(want)).to(F32).to(odt)      # (rounded to float, then to the type, as the product is)
        assert torch.equal(got.cpu(), once) and torch.equal(torch.signbit(got.cpu()), torch.signbit(once))


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_matrices(block_rows):
    """Blocks of 128 rows end with their matrix; several dimensions of either kind."""
    x = normal((3, 130, 4, 40), 5, F32, spread=3.0)
    m = gs.f8_quantize(x.to(DEV), n_access=2, block_rows=block_rows)
    code, scales = f8.quantize(to_oracle(x).reshape(3, 130, 160), block_rows)
    assert np.array_equal(codes_of(m), code)
    same_scales(m.scales, scales)
    got = gs.f8_dequantize(m, out_dtype=F32)
    assert np.array_equal(to_oracle(got).reshape(3, 130, 160), f8.round32(f8.dequantize(code, scales, 160, block_rows)))


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape", [(), (5,), (300,), (3, 100)])
def test_quantize_one_element(shape, block_rows):
    """Every dimension a compute dimension; a number by itself."""
    x = normal(shape, 7, F32) if shape else torch.tensor(-3.7)
    m = gs.f8_quantize(x.to(DEV), n_access=0, block_rows=block_rows)
    code, scales = f8.quantize(to_oracle(x).reshape(1, 1, -1), block_rows)
    assert m.values.shape == code.shape[2:] and np.array_equal(codes_of(m), code[0, 0])
    same_scales(m.scales, scales[0, 0])
    assert np.array_equal(to_oracle(gs.f8_dequantize(m, out_dtype=F32)).reshape(-1), f8.round32(f8.dequantize(code, scales, x.numel(), block_rows))[0, 0])


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_nothing(block_rows):
    for shape in ((0, 64), (4, 0), (0, 0), (2, 0, 5), (0, 3, 5)):
        m = gs.f8_quantize(torch.zeros(shape, device=DEV), block_rows=block_rows)
        assert m.values.numel() == 0 and gs.f8_dequantize(m).shape == shape
        assert gs.norm(torch.zeros(shape, device=DEV))[0].shape == shape and gs.f8_norm(torch.zeros(shape, device=DEV))[0].shape == shape


def test_quantize_many():
    """More pieces than a lane's first, rows of every alignment."""
    for rows, cols, dtype in ((4100, 1025, BF), (2051, 2050, F32)):
        x = normal((rows, cols), rows, dtype, spread=2.0)
        m = gs.f8_quantize(x.to(DEV))
        code, scales = f8.quantize(to_oracle(x)[None])
        assert np.array_equal(codes_of(m), code[0])
        same_scales(m.scales, scales[0])
        assert np.array_equal(to_oracle(gs.f8_dequantize(m, out_dtype=F32)), f8.round32(f8.dequantize(code, scales, cols))[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_borders(dtype):
    """Every border between codes and its neighbours, at scales from the smallest to the largest."""
    both = np.sort(np.concatenate((f8.CODES[:127], (f8.CODES[1:127] + f8.CODES[:126]) / 2)))
    rows = []
    for e in (-149, -134, -130, -126, -118, -20, -1, 0, 1, 20, 100, 118):
        for part in np.split(both, range(100, len(both), 100)):
            row = np.zeros(128)
            row[0] = 448.0
            row[1:1 + len(part)] = part
            rows += [row * 2.0 ** e, -row * 2.0 ** e, np.nextafter(np.float32(row), np.float32(0)) * 2.0 ** e]
    x = torch.from_numpy(np.stack(rows)).to(dtype)
    m = gs.f8_quantize(x.to(DEV))
    code, scales = f8.quantize(to_oracle(x)[None])
    same_scales(m.scales, scales[0])
    assert np.array_equal(codes_of(m), code[0])


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_infinities_and_nan(dtype, block_rows):
    x = normal((260, 260), 9, dtype)
    x[0, 0], x[130, 129], x[255, 259] = float("inf"), float("nan"), float("-inf")
    m = gs.f8_quantize(x.to(DEV), block_rows=block_rows)
    code, scales = f8.quantize(to_oracle(x)[None], block_rows)
    assert np.isnan(scales).sum() == 3
    assert np.array_equal(codes_of(m), code[0])
    same_scales(m.scales, scales[0])
    want = f8.round32(f8.dequantize(code, scales, 260, block_rows)[0])
    assert np.array_equal(to_oracle(gs.f8_dequantize(m, out_dtype=F32)), want, equal_nan=True)


def test_largest_numbers():
    x = torch.tensor([[3.3895e38, -3.3895e38, 1.0, 1e-45]], dtype=F32)
    m = gs.f8_quantize(x.to(DEV))
    code, scales = f8.quantize(to_oracle(x)[None])
    assert np.array_equal(codes_of(m), code[0])
    same_scales(m.scales, scales[0])


def test_dequantize_every_code():
    values = torch.arange(256, dtype=torch.uint8).view(2, 1, 128).to(DEV)
    scales = torch.tensor([[0.37, 0, 0, 0], [2.0 ** -120, 0, 0, 0]], device=DEV)
    m = gs.F8(values, scales, (2, 128), 1, 1)
    want = f8.round32(f8.dequantize(values.cpu().numpy()[None], to_oracle(scales)[None], 128)[0])
    assert np.array_equal(to_oracle(gs.f8_dequantize(m, out_dtype=F32)), want, equal_nan=True)


def test_quantize_into():
    x = normal((5, 300), 3).to(DEV)
    m = gs.f8_quantize(x)
    values, scales = torch.full((5 * 3 * 128 + 100,), 7, dtype=torch.uint8, device=DEV), torch.full((5 * 4 + 9,), 7.0, device=DEV)
    out = gs.F8(values[:5 * 3 * 128].view(5, 3, 128), scales[:20].view(5, 4), (5, 300), 1, 1)
    assert gs.f8_quantize(x, out=out) is out
    assert torch.equal(out.values, m.values.view(torch.uint8)) and torch.equal(out.scales, m.scales)
    assert (values[5 * 3 * 128:] == 7).all() and (scales[20:] == 7).all()
    flat = torch.full((5 * 300 + 64,), 7, dtype=BF, device=DEV)
    gs.f8_dequantize(m, out=flat[:1500].view(5, 300))
    assert torch.equal(flat[:1500].view(5, 300), gs.f8_dequantize(m)) and (flat[1500:] == 7).all()


# ------------------------------------------------------------------------------------------------
# norms
# ------------------------------------------------------------------------------------------------

NORM_COLS = [1, 7, 100, 128, 129, 512, 513, 1024, 1025, 2048, 2050, 4096, 4099, 8192, 8200, 16384, 16392, 40000]


@pytest.mark.parametrize("wdt", [None, BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cols", NORM_COLS)
def test_norm(cols, dtype, wdt):
    rows = 1 if cols > 16384 else 9
    x, res = normal((rows, cols), cols, dtype, 3.0), normal((rows, cols), cols + 1, dtype, 3.0)
    weight = None if wdt is None else (1 + 0.3 * normal((cols,), 5, F32)).to(wdt)
    on = None if weight is None else weight.to(DEV)
    for residual in (None, res):
        h = x if residual is None else (x.float() + residual.float()).to(dtype)
        want = f8.norm(to_oracle(h), None if weight is None else to_oracle(weight), np.float64(np.float32(1e-5)))
        more = None if residual is None else residual.to(DEV)
        for odt in (BF, F32):
            got, total = gs.norm(x.to(DEV), on, residual=more, eps=1e-5, out_dtype=odt)
            assert got.dtype == odt and torch.equal(total.cpu(), h)
            assert torch.equal(got.cpu(), torch.from_numpy(f8.round32(want)).to(F32).to(odt))
        m, total = gs.f8_norm(x.to(DEV), on, residual=more, eps=1e-5)
        assert torch.equal(total.cpu(), h) and m.shape == (rows, cols) and m.block_rows == 1
        code, scales = f8.quantize(f8.round32(want)[None])
        assert np.array_equal(codes_of(m), code[0])
        same_scales(m.scales, scales[0])


@pytest.mark.parametrize("cols", [32768, 32769, 50007])
def test_norm_of_several_long_rows(cols):
    """Rows that registers hold no longer are read twice."""
    x, res, w = normal((5, cols), 1), normal((5, cols), 2), normal((cols,), 3, F32)
    h = (x.float() + res.float()).to(BF)
    want = f8.norm(to_oracle(h), to_oracle(w), np.float64(np.float32(1e-5)))
    got, total = gs.norm(x.to(DEV), w.to(DEV), residual=res.to(DEV), eps=1e-5, out_dtype=F32)
    assert torch.equal(total.cpu(), h) and torch.equal(got.cpu(), torch.from_numpy(f8.round32(want)).to(F32))
    m, total = gs.f8_norm(x.to(DEV), w.to(DEV), residual=res.to(DEV), eps=1e-5)
    code, scales = f8.quantize(f8.round32(want)[None])
    assert torch.equal(total.cpu(), h) and np.array_equal(codes_of(m), code[0])
    same_scales(m.scales, scales[0])


def test_norm_is_that_of_the_sum_as_stored():
    x, res, w = normal((17, 1000), 1).to(DEV), normal((17, 1000), 2).to(DEV), normal((1000,), 3).to(DEV)
    total = gs.pair_reduce(x, res)
    for f in (gs.norm, gs.f8_norm):
        a, sum_a = f(x, w, residual=res)
        b, sum_b = f(total, w)
        assert torch.equal(sum_a, total) and sum_b.data_ptr() == total.data_ptr()
        for u, v in zip(a if isinstance(a, gs.F8) else (a,), b if isinstance(b, gs.F8) else (b,)):
            if isinstance(u, torch.Tensor):
                assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))
        given = torch.empty_like(x)
        _, out = f(x, w, total=given)
        assert out is given and torch.equal(given, x)


def test_f8_norm_is_the_norm_quantised():
    """A float result, quantised afterwards, is the same bit for bit."""
    x, w = normal((33, 1300), 1, F32, 4.0).to(DEV), normal((1300,), 3, F32).to(DEV)
    y, _ = gs.norm(x, w, eps=1e-6)
    a, (b, _) = gs.f8_quantize(y), gs.f8_norm(x, w, eps=1e-6)
    assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)


def test_norm_several_dimensions():
    x, w = normal((3, 4, 5, 60), 1).to(DEV), normal((5, 60), 2).to(DEV)
    y, _ = gs.norm(x, w, n_access=2)
    want = f8.norm(to_oracle(x).reshape(12, 300), to_oracle(w).reshape(300), 1e-6).reshape(3, 4, 5, 60)
    within(y, want, np.abs(want) * (2.0 ** -24 + 2.0 ** -8) * (1 + 2.0 ** -7))


def test_norm_of_zeros_and_infinities():
    x = torch.zeros(4, 300)
    x[1, 7], x[2, 299] = float("inf"), float("nan")
    x[3] = 1.0
    y, _ = gs.norm(x.to(DEV))
    m, _ = gs.f8_norm(x.to(DEV))
    y, scales, code = to_oracle(y), to_oracle(m.scales), codes_of(m)
    assert (y[0] == 0).all() and np.isnan(y[1, 7]) and (np.delete(y[1], 7) == 0).all() and np.isnan(y[2]).all()
    assert np.isnan(scales[1, 0]) and (scales[1, 1:3] == 2.0 ** -126).all() and np.isnan(scales[2, :3]).all()
    assert (scales[:, 3] == 0).all() and not code[0].any() and not code[2].any()
    # the largest and the smallest numbers: no square is lost
    x = torch.stack((torch.full((300,), 3e38), torch.full((300,), 1e-38), torch.full((300,), 1e-44)))
    x[:, 0] = 0
    y, _ = gs.norm(x.to(DEV), eps=0.0)
    want = f8.norm(to_oracle(x), None, 0.0)
    assert np.array_equal(to_oracle(y), f8.round32(want)) and want.max() < 1.01
    # rows without anything: the root is of eps alone
    y, _ = gs.norm(torch.zeros(2, 300, device=DEV), eps=0.0)
    assert torch.isnan(y).all()


# ------------------------------------------------------------------------------------------------
# products
# ------------------------------------------------------------------------------------------------


def operand(shape, n_access, block_rows, seed, spread=2.0):
    """An F8 pattern on the GPU, and its numbers as (mats, rows, K)."""
    x = normal(shape, seed, F32, spread)
    m = gs.f8_quantize(x.to(DEV), n_access=n_access, block_rows=block_rows)
    rows = shape[n_access - 1] if n_access else 1
    mats = int(np.prod(shape[:max(n_access - 1, 0)]))
    cols = int(np.prod(shape[n_access:]))
    blocks, groups = -(-cols // 128), -(-rows // block_rows)
    return m, f8.dequantize(codes_of(m).reshape(mats, rows, blocks, 128), to_oracle(m.scales).reshape(mats, groups, -1), cols, block_rows)


def allowed(size, want, blocks, odt):
    slack = size * (2.0 ** -13 + (blocks + 2) * 2.0 ** -24)
    return slack + (np.abs(want) + slack) * EPS[odt] + 1e-37


def check_dot(m, n, k, x_rows=1, w_rows=128, odt=BF, act=gs.GS_ACT_NONE, seed=0):
    (x, xv), (w, wv) = operand((m, k), 1, x_rows, 11 + seed), operand((n, k), 1, w_rows, 12 + seed)
    got = gs.f8_dot(x, w, out_dtype=odt, act=act)
    assert got.shape == (m, n) and got.dtype == odt
    want, size = xv[0] @ wv[0].T, np.abs(xv[0]) @ np.abs(wv[0]).T
    if act == gs.GS_ACT_RELU:
        want = np.maximum(want, 0)
    within(got, want, allowed(size, want, -(-k // 128), odt))


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("k", [1, 128, 130, 513, 1000, 2048, 4100])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 300), (3, 16), (16, 130), (17, 33), (40, 257), (64, 64)])
def test_dot_few(m, n, k, w_rows):
    check_dot(m, n, k, w_rows=w_rows, odt=F32 if k % 2 else BF)


@pytest.mark.parametrize("x_rows", [1, 128])
@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("m,n,k", [(100, 1000, 700), (257, 513, 384), (300, 200, 1100), (129, 129, 128), (511, 770, 2050), (700, 1300, 130), (1100, 1290, 300)])
def test_dot_many(m, n, k, x_rows, w_rows):
    check_dot(m, n, k, x_rows, w_rows)


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("m,n,k", [(2, 70, 300), (200, 300, 300), (300, 2100, 260)])
def test_dot_relu_and_floats(m, n, k, w_rows):
    check_dot(m, n, k, w_rows=w_rows, act=gs.GS_ACT_RELU, seed=5)
    check_dot(m, n, k, w_rows=w_rows, odt=F32, seed=6)


@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("m,n,k", [(5, 200, 1000), (130, 260, 520), (260, 1300, 1030), (1030, 2060, 640)])
def test_dot_exactly(m, n, k, w_rows):
    """Small whole numbers with scales of powers of two: every sum is exact, whatever its order, and a number in a wrong place shows."""
    g = torch.Generator().manual_seed(m)
    xc, wc = torch.randint(-3, 4, (m, k), generator=g), torch.randint(-3, 4, (n, k), generator=g)
    blocks, run = -(-k // 128), -(-k // 512) * 4
    xs = torch.exp2(torch.randint(0, 3, (m, run), generator=g).float())
    ws = torch.exp2(torch.randint(0, 3, (-(-n // w_rows), run), generator=g).float())

    def codes(c):
        return torch.nn.functional.pad(c.float(), (0, blocks * 128 - k)).to(torch.float8_e4m3fn).view(c.shape[0], blocks, 128)

    x, w = gs.F8(codes(xc).to(DEV), xs.to(DEV), (m, k), 1, 1), gs.F8(codes(wc).to(DEV), ws.to(DEV), (n, k), 1, w_rows)
    xv = (codes(xc).double() * xs[:, :blocks, None].double()).flatten(1)
    wv = (codes(wc).double() * ws.repeat_interleave(w_rows, 0)[:n, :blocks, None].double()).flatten(1)
    want = xv @ wv.t()
    assert want.abs().max() < 2 ** 24
    assert torch.equal(gs.f8_dot(x, w, out_dtype=F32).cpu().double(), want)


def test_dot_dimensions():
    (x, xv), (w, wv) = operand((2, 3, 4, 50), 2, 1, 1), operand((128, 4, 50), 1, 128, 2)
    got = gs.f8_dot(x, w)
    want, size = xv.reshape(6, 200) @ wv[0].T, np.abs(xv.reshape(6, 200)) @ np.abs(wv[0]).T
    assert got.shape == (2, 3, 128) and got.dtype == F32
    within(got.reshape(6, 128), want, allowed(size, want, 2, F32))
    # a matrix of two access dimensions in blocks of 128 rows, the last of them whole blocks
    (w, wv) = operand((2, 128, 200), 2, 128, 3)
    (x, xv) = operand((5, 200), 1, 1, 4)
    got = gs.f8_dot(x, w)
    want, size = xv[0] @ wv.reshape(256, 200).T, np.abs(xv[0]) @ np.abs(wv.reshape(256, 200)).T
    assert got.shape == (5, 2, 128)
    within(got.reshape(5, 256), want, allowed(size, want, 2, F32))


@pytest.mark.parametrize("m", [2, 40])
def test_dot_of_the_longest_rows(m):
    """Beyond 2^22 numbers, where few of them are not zero: sums are exact."""
    k, n = (1 << 22) + 300, 33
    blocks = -(-k // 128)
    g = torch.Generator(device=DEV).manual_seed(1)
    x, w = (torch.where(torch.rand(r, k, generator=g, device=DEV) < 2e-3, torch.randint(-3, 4, (r, k), generator=g, device=DEV).float(), 0.0) for r in (m, n))
    x[:, -1], w[:, -1] = 2.0, 3.0

    def held(t):
        codes = torch.nn.functional.pad(t, (0, blocks * 128 - k)).to(torch.float8_e4m3fn).view(t.shape[0], blocks, 128)
        return gs.F8(codes, torch.ones(t.shape[0], -(-blocks // 4) * 4, device=DEV), tuple(t.shape), 1, 1)

    assert torch.equal(gs.f8_dot(held(x), held(w)), x @ w.t().contiguous())


@pytest.mark.parametrize("m", [3, 300])
def test_dot_without_anything(m):
    x, w = gs.f8_quantize(torch.zeros(m, 0, device=DEV)), gs.f8_quantize(torch.zeros(70, 0, device=DEV), block_rows=128)
    out = torch.full((m, 70), 3.0, device=DEV)
    assert not gs.f8_dot(x, w, out=out).any()
    x, w = gs.f8_quantize(torch.zeros(0, 64, device=DEV)), gs.f8_quantize(torch.zeros(70, 64, device=DEV), block_rows=128)
    assert gs.f8_dot(x, w).shape == (0, 70)


@pytest.mark.parametrize("m,n", [(2, 40), (300, 300)])
def test_dot_nan_and_infinities(m, n):
    """A NaN is that of its row or column alone; so is a block whose scales are too large together."""
    x, w = normal((m, 300), 1, F32), normal((n, 300), 2, F32)
    x[1, 200] = float("inf")
    w[n - 1, 5] = float("nan")
    a, b = gs.f8_quantize(x.to(DEV)), gs.f8_quantize(w.to(DEV))
    got = gs.f8_dot(a, b)
    nan = torch.isnan(got).cpu()
    assert nan[1].all() and nan[:, n - 1].all() and nan.sum() == m + n - 1
    big = gs.F8(b.values, torch.where(torch.isnan(b.scales), 1.0, b.scales).fill_(1e38), (n, 300), 1, 1)
    few = gs.F8(a.values, torch.full_like(a.scales, 1e-30), (m, 300), 1, 1)
    assert torch.isfinite(gs.f8_dot(few, big)).all()


def test_dot_twice_is_the_same():
    (x, _), (w, _) = operand((333, 2000), 1, 1, 1), operand((700, 2000), 1, 128, 2)
    assert torch.equal(gs.f8_dot(x, w), gs.f8_dot(x, w))
