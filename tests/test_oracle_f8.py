"""The oracle of scaled 8-bit floats, norms and experts, pinned: to torch's own conversion to e4m3, to hand-computed values, and to other
ways of computing the same."""

import numpy as np
import pytest
import torch

from oracle import f8, numerics


def test_codes_ascend_and_end_at_448():
    assert f8.CODES[0] == 0 and f8.CODES[1] == 2.0 ** -9 and f8.CODES[8] == 2.0 ** -6 and f8.CODES[126] == 448 and np.isnan(f8.CODES[127])
    assert (np.diff(f8.CODES[:127]) > 0).all()


def test_nearest_code_is_torchs_conversion():
    """Every border, both neighbours in float, and many between."""
    mid = (f8.CODES[1:127] + f8.CODES[:126]) / 2
    x = np.concatenate((f8.CODES[:127], mid, np.nextafter(np.float32(mid), np.float32(0)), np.nextafter(np.float32(mid), np.float32(500)),
                        np.random.default_rng(1).uniform(0, 448, 20000), np.exp2(np.random.default_rng(2).uniform(-14, 8.8, 20000))))
    x = np.minimum(np.float32(x), np.float32(448))
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(f8.nearest_code(x), want)


def test_quantize_by_hand():
    x = np.zeros((1, 2, 130))
    x[0, 0, 0], x[0, 0, 1], x[0, 0, 128], x[0, 1, 0] = 448.0, -1.0, 7.0, -896.0
    code, scales = f8.quantize(x)
    assert code.shape == (1, 2, 2, 128) and scales.shape == (1, 2, 4)
    s = [float(np.float32(v) * np.float32(1 / 448)) for v in (448.0, 7.0, 896.0)]
    assert np.array_equal(scales[0], [[s[0], s[1], 0, 0], [s[2], 2.0 ** -126, 0, 0]])
    assert code[0, 0, 0, 0] == 126 and code[0, 0, 0, 1] == 128 + 56 and code[0, 0, 1, 0] == 126 and code[0, 1, 0, 0] == 254 and code[0, 0, 1, 2] == 0
    code, scales = f8.quantize(x, 128)
    assert scales.shape == (1, 1, 4) and scales[0, 0, 0] == s[2] and code[0, 0, 0, 0] == f8.nearest_code(224.0)
    back = f8.dequantize(code, scales, 130, 128)
    assert back.shape == x.shape and abs(back[0, 0, 0] - 448) <= 448 * 2.0 ** -20


def test_quantize_is_within_half_a_step():
    x = np.random.default_rng(3).standard_normal((2, 200, 300)) * 10.0
    for rows in (1, 128):
        code, scales = f8.quantize(x, rows)
        of = np.repeat(np.repeat(scales[:, :, :3], rows, 1)[:, :200], 128, 2)[:, :, :300]
        err = np.abs(f8.dequantize(code, scales, 300, rows) - x)
        assert (err <= np.maximum(np.abs(x) * 2.0 ** -4, of * 2.0 ** -10) * (1 + 2.0 ** -20)).all()
        assert np.array_equal(f8.quantize(f8.dequantize(code, scales, 300, rows), rows)[0], code)


def test_quantize_what_is_broken():
    x = np.ones((1, 130, 260))
    x[0, 3, 5], x[0, 129, 259] = np.inf, np.nan
    code, scales = f8.quantize(x)
    assert np.isnan(scales[0, 3, 0]) and np.isnan(scales[0, 129, 2]) and np.isnan(scales).sum() == 2 and not code[0, 3, 0].any()
    code, scales = f8.quantize(x, 128)
    assert np.isnan(scales[0, 0, 0]) and np.isnan(scales[0, 1, 2]) and np.isnan(scales).sum() == 2


def test_norm_is_torchs():
    x, w = np.random.default_rng(4).standard_normal((5, 70)), np.random.default_rng(5).standard_normal(70)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (70,), torch.from_numpy(w), 1e-5).numpy()
    assert np.allclose(f8.norm(x, w, 1e-5), want, rtol=1e-12) and np.allclose(f8.norm(x, None, 1e-5) * w, want, rtol=1e-12)


@pytest.mark.parametrize("tokens,choices,experts", [(0, 2, 3), (1, 1, 1), (40, 3, 5)])
def test_sort_is_a_stable_sort(tokens, choices, experts):
    e = np.random.default_rng(6).integers(-1, experts + 1, (tokens, choices))
    offsets, of, places = f8.sort(e, experts)
    flat = e.reshape(-1)
    kept = np.nonzero((flat >= 0) & (flat < experts))[0]
    order = kept[np.argsort(flat[kept], kind="stable")]
    assert np.array_equal(offsets, np.searchsorted(flat[order], np.arange(experts + 1)))
    assert np.array_equal(of[:len(order)], order // choices) and (of[len(order):] == -1).all()
    assert np.array_equal(places.reshape(-1)[order], np.arange(len(order))) and (places >= 0).sum() == len(order)


def test_rows_are_products_with_a_matrix():
    """Spreading out and joining are linear: P x and (P with weights)^T y, and the gradients those of autograd."""
    rng = np.random.default_rng(7)
    e = rng.integers(-1, 4, (9, 3))
    _, _, places = f8.sort(e, 4)
    x, rows, weights, grad = rng.standard_normal((9, 5)), rng.standard_normal((27, 5)), rng.standard_normal((9, 3)), rng.standard_normal((9, 5))
    spread = f8.split(x, places, rows)
    p = torch.from_numpy(places)
    r, w = torch.from_numpy(rows).requires_grad_(), torch.from_numpy(weights).requires_grad_()
    y = (torch.where((p >= 0)[..., None], r[p.clamp(min=0)], 0.0) * w[..., None]).sum(1)
    assert np.allclose(f8.join(rows, places, weights)[0], y.detach().numpy())
    y.backward(torch.from_numpy(grad))
    grad_rows, grad_weights, _ = f8.join_grad(grad, rows, places, weights, np.zeros_like(rows))
    assert np.allclose(grad_rows, r.grad.numpy()) and np.allclose(grad_weights, w.grad.numpy())
    # <split(x), y> = <x, join(y)> where all rows are somebody's or zero
    zero = f8.split(x, places, np.zeros_like(rows))
    assert np.isclose((zero * rows).sum(), (x * f8.join(rows, places, None)[0]).sum())
    assert np.array_equal(spread[zero.any(1)], zero[zero.any(1)])


def test_expert_dot_by_hand():
    x, w = np.arange(6.0).reshape(3, 2), np.arange(8.0).reshape(2, 2, 2)
    out, size = f8.expert_dot(x, np.array([2, -1, 0, 1]), [0, 2, 3], w, np.full((4, 2), 9.0))
    assert out.tolist() == [[5, 23], [0, 0], [5, 7], [9, 9]] and size[3].tolist() == [0, 0]
    assert numerics.round_to_f32(out).tolist() == out.tolist()
