"""Pins of the oracle of microscaled 4-bit floats: values by hand, the format's tables, closed forms."""

import numpy as np
import pytest
import torch

from oracle import mx4


def test_every_code_and_scale():
    want = [0, .5, 1, 1.5, 2, 3, 4, 6]
    assert list(mx4.E2M1[:8]) == want and list(mx4.E2M1[8:]) == [-w for w in want]
    # sign, two bits of exponent (bias 1), one of mantissa
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        v = (m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)) * (-1) ** (c >> 3)
        assert mx4.E2M1[c] == v
    assert mx4.scale_value(127) == 1 and mx4.scale_value(0) == 2.0 ** -127 and np.isnan(mx4.scale_value(255))
    bits = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(mx4.scale_value(bits.numpy()), bits.view(torch.float8_e8m0fnu).to(torch.float64).numpy(), equal_nan=True)


@pytest.mark.parametrize("a,code", [(0.25, 0), (0.2500001, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.01, 7),
                                    (7.99, 7), (100.0, 7), (0.0, 0), (0.74, 1)])
def test_rounding_by_hand(a, code):
    assert mx4.nearest_code(a) == code


def test_scale_by_hand():
    for top, byte in ((4.0, 127), (7.9, 127), (3.99, 126), (8.0, 128), (1.0, 125), (0.0, 0), (2.0 ** -126, 0), (2.0 ** -149, 0), (2.0 ** 127, 252)):
        x = np.zeros((1, 32))
        x[0, 7] = -top
        packed, scales = mx4.quantize(x)
        assert scales[0, 0] == byte, top
        assert not scales[0, 1:].any()
        back = mx4.dequantize(packed, scales, 32)
        if top in (4.0, 8.0, 1.0, 2.0 ** -126, 2.0 ** 127):       # representable
            assert back[0, 7] == -top


def test_numbers_of_the_format_survive():
    rng = np.random.default_rng(5)
    code = rng.integers(0, 16, (7, 100))
    code[:, ::32] = 7                                       # a six in every block: the scale is found again
    x = mx4.E2M1[code] * 8.0
    packed, scales = mx4.quantize(x)
    assert np.array_equal(mx4.dequantize(packed, scales, 100), x)
    assert packed.shape == (7, 4, 16) and scales.shape == (7, 8) and not packed[:, 3, 2:].any()


def test_infinities_and_nan_break_their_block_only():
    x = np.ones((1, 96))
    x[0, 5], x[0, 40] = np.inf, np.nan
    packed, scales = mx4.quantize(x)
    back = mx4.dequantize(packed, scales, 96)
    assert np.isnan(back[0, :64]).all() and (back[0, 64:] == 1).all()


@pytest.mark.parametrize("page,dim", [(16, 64), (48, 96), (64, 128), (32, 256)])
def test_cache_layout_is_a_bijection(page, dim):
    seen = np.concatenate([np.concatenate(mx4.token_offsets(page, dim, s)) for s in range(page)])
    assert sorted(seen) == list(range(mx4.block_bytes(page, dim)))


def test_attention_of_equal_keys_is_the_mean():
    rng = np.random.default_rng(6)
    page, dim, n = 16, 64, 21
    data = np.zeros((3, 1, mx4.block_bytes(page, dim)), np.uint8)
    table = np.array([[2, 0]], np.int32)
    v = rng.standard_normal((1, n, 1, dim))
    mx4.append(data, table, [0], None, np.ones((1, n, 1, dim)), v, page, dim)
    vq = mx4.dequantize(*mx4.quantize(v[0, :, 0]), dim)
    out, _ = mx4.attend(rng.standard_normal((1, 2, 1, dim)), data, table, [n], page, 0.3)
    assert np.allclose(out[0, 1, 0], vq.mean(0)) and np.allclose(out[0, 0, 0], vq[:-1].mean(0))
    out, _ = mx4.attend(rng.standard_normal((1, 1, 1, dim)), data, table, [n], page, 0.3, window=3, sinks=2)
    assert np.allclose(out[0, 0, 0], vq[[0, 1, n - 3, n - 2, n - 1]].mean(0))
