"""Scaled 8-bit floats, root-mean-square norms and tokens dealt to experts, from their definitions.  Plain numpy, one step at a time;
what the definitions round to float is rounded to float here, the rest is float64."""

import numpy as np

from oracle import numerics

BLOCK = 128
LEAST = np.float64(2.0 ** -126)
UNIT = np.float64(np.float32(1.0 / 448.0))
CODES = numerics.e4m3_bits_to_f64(np.arange(128))        # of the positive numbers, ascending; the last is NaN


def round32(x):
    with np.errstate(over="ignore", invalid="ignore"):
        return np.asarray(x, dtype=np.float64).astype(np.float32).astype(np.float64)


def nearest_code(a):
    """The e4m3 code nearest to a magnitude of at most 448, ties to the even code."""
    a = np.asarray(a, dtype=np.float64)
    up = np.clip(np.searchsorted(CODES[:127], a), 1, 126)
    low, high = a - CODES[up - 1], CODES[up] - a
    return np.where((low < high) | ((low == high) & (up % 2 == 1)), up - 1, up)


def scale_of(top, broken):
    s = np.maximum(round32(np.where(broken, 0.0, top) * UNIT), LEAST)
    return np.where(broken, np.nan, s)


def quantize(x, block_rows=1):
    """(mats, rows, K) float64 -> codes (mats, rows, B, 128), scales (mats, rows / block_rows, B up to a multiple of 4)."""
    x = np.asarray(x, dtype=np.float64)
    mats, rows, k = x.shape
    blocks, groups = -(-k // BLOCK), -(-rows // block_rows)
    wide = np.zeros((mats, groups * block_rows, blocks * BLOCK))
    wide[:, :rows, :k] = x
    wide = wide.reshape(mats, groups, block_rows, blocks, BLOCK)
    finite = np.isfinite(wide)
    broken = ~finite.all((2, 4))
    clean = np.where(broken[:, :, None, :, None], 0.0, wide)
    scale = scale_of(np.abs(clean).max((2, 4), initial=0.0), broken)
    factor = round32(1.0 / np.where(broken, 1.0, scale))
    code = nearest_code(np.abs(round32(clean * factor[:, :, None, :, None]))) + 128 * np.signbit(clean)
    code = np.where(broken[:, :, None, :, None], 0, code)
    code = code.reshape(mats, groups * block_rows, blocks, BLOCK)[:, :rows].astype(np.uint8)
    padded = np.zeros((mats, groups, -(-blocks // 4) * 4))
    padded[:, :, :blocks] = scale
    return code, padded


def dequantize(code, scales, k, block_rows=1):
    """The numbers (mats, rows, K), not rounded."""
    mats, rows, blocks = code.shape[:3]
    s = np.repeat(scales, block_rows, 1)[:, :rows, :blocks]
    with np.errstate(invalid="ignore"):
        return (numerics.e4m3_bits_to_f64(code) * s[..., None]).reshape(mats, rows, -1)[:, :, :k]


def norm(h, weight, eps):
    """(rows, K) -> the norm, not rounded."""
    y = h / np.sqrt((h * h).sum(1, keepdims=True) / h.shape[1] + eps)
    return y if weight is None else y * weight


def sort(experts, n_experts):
    """(T, choices) -> offsets, tokens, places."""
    places = np.full(experts.shape, -1, dtype=np.int64)
    tokens = np.full(experts.size, -1, dtype=np.int64)
    offsets, row = [0], 0
    for e in range(n_experts):
        for t, j in zip(*np.nonzero(experts == e)):
            places[t, j], tokens[row] = row, t
            row += 1
        offsets.append(row)
    return np.array(offsets), tokens, places


def split(x, places, rows):
    rows = rows.copy()
    for t, j in zip(*np.nonzero((places >= 0) & (places < len(rows)))):
        rows[places[t, j]] = x[t]
    return rows


def join(rows, places, weights):
    """-> the sums, and the sums of their terms' magnitudes."""
    out = np.zeros((len(places),) + rows.shape[1:])
    size = np.zeros_like(out)
    for t, j in zip(*np.nonzero((places >= 0) & (places < len(rows)))):
        term = rows[places[t, j]] * (1.0 if weights is None else weights[t, j])
        out[t] += term
        size[t] += np.abs(term)
    return out, size


def join_grad(grad, rows, places, weights, grad_rows):
    """-> the rows' gradients, the weights', and the sums of the magnitudes of the latter's terms."""
    grad_rows = grad_rows.copy()
    grad_weights, size = np.zeros(places.shape), np.zeros(places.shape)
    for t, j in zip(*np.nonzero((places >= 0) & (places < len(rows)))):
        p = places[t, j]
        grad_rows[p] = grad[t] * (1.0 if weights is None else weights[t, j])
        grad_weights[t, j] = (grad[t] * rows[p]).sum()
        size[t, j] = np.abs(grad[t] * rows[p]).sum()
    return grad_rows, grad_weights, size


def expert_dot(x, tokens, offsets, w, out):
    """Rows of x (T, K) by tokens, w (E, N, K) -> out, and the sums of the terms' magnitudes (zero where nothing is written)."""
    out = out.copy()
    size = np.zeros_like(out)
    m = len(out)
    lo = min(max(int(offsets[0]), 0), m)
    for e in range(len(w)):
        hi = max(lo, min(int(offsets[e + 1]), m))            # (no offset is taken as below one before it)
        for r in range(lo, hi):
            t = r if tokens is None else int(tokens[r])
            row = x[t] if 0 <= t < len(x) else np.zeros(w.shape[2])
            out[r] = w[e] @ row
            size[r] = np.abs(w[e]) @ np.abs(row)
        lo = hi
    return out, size
