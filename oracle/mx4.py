"""Microscaled 4-bit floats from the format's definition, in float64: e2m1 numbers in blocks of 32 with an e8m0 scale,
the layout of the paged cache, and attention over it.  Plain numpy, one step at a time."""

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])
BLOCK = 32


def scale_value(byte):
    """e8m0: 2^(byte - 127), 255 is NaN."""
    byte = np.asarray(byte, dtype=np.int64)
    return np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))


def nearest_code(a):
    """Code of the e2m1 value nearest to a magnitude, ties to the even code, above 6 the largest."""
    a = np.asarray(a, dtype=np.float64)
    d = np.abs(a[..., None] - E2M1[:8])
    best = d.min(-1, keepdims=True)
    is_best = d == best
    order = np.where(is_best, np.arange(8) % 2 * 8 + np.arange(8), 99)      # even codes in front of odd ones
    return order.argmin(-1)


def quantize(x):
    """(rows, K) float64 -> codes' bytes (rows, B, 16), scale bytes (rows, B up to a multiple of 8)."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    blocks = -(-k // BLOCK)
    padded = np.zeros((rows, blocks * BLOCK))
    padded[:, :k] = x
    padded = padded.reshape(rows, blocks, BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.abs(padded).max(-1)
    broken = ~np.isfinite(padded).all(-1)
    safe = np.where(broken | (top == 0), 1.0, top)
    e = np.floor(np.log2(safe)).astype(np.int64)
    e = np.where(np.ldexp(1.0, e) > safe, e - 1, e)
    e = np.where(np.ldexp(1.0, e + 1) <= safe, e + 1, e)
    byte = np.clip(e - 2 + 127, 0, 254)
    byte = np.where(top == 0, 0, byte)
    clean = np.where(broken[..., None], 0.0, padded)
    code = nearest_code(np.abs(clean) / np.ldexp(1.0, byte - 127)[..., None])
    code = code + 8 * np.signbit(clean)
    code = np.where(broken[..., None], 0, code)
    byte = np.where(broken, 255, byte)
    packed = (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)
    scales = np.zeros((rows, -(-blocks // 8) * 8), dtype=np.uint8)
    scales[:, :blocks] = byte
    return packed, scales


def dequantize(packed, scales, k):
    """(rows, B, 16), (rows, >= B) -> (rows, K) float64."""
    packed = np.asarray(packed)
    rows, blocks = packed.shape[:2]
    code = np.stack((packed & 15, packed >> 4), -1).reshape(rows, blocks, BLOCK)
    with np.errstate(invalid="ignore"):
        v = E2M1[code] * scale_value(scales[:, :blocks])[..., None]
    return v.reshape(rows, -1)[:, :k]


def block_bytes(page, dim):
    return page * dim + 2 * page * (dim // BLOCK)


def token_offsets(page, dim, slot):
    """Byte offsets in a (page, head) block: key (D/2), value (D/2), key scales (D/32), value scales (D/32)."""
    half, few = page * dim // 2, page * dim // BLOCK
    key = slot * (dim // 2) + np.arange(dim // 2)
    piece, byte = np.divmod(np.arange(dim // 2), 4)
    value = half + ((slot // 4) * (dim // 8) + piece) * 16 + (slot % 4) * 4 + byte
    key_scale = 2 * half + slot * (dim // BLOCK) + np.arange(dim // BLOCK)
    value_scale = 2 * half + few + ((slot // 4) * (dim // BLOCK) + np.arange(dim // BLOCK)) * 4 + slot % 4
    return key, value, key_scale, value_scale


def place(table_row, n_pages, page, t):
    """(page id, slot) of a token, or None where it has no page."""
    if t < 0 or t >= len(table_row) * page:
        return None
    pid = int(table_row[t // page])
    return (pid, t % page) if 0 <= pid < n_pages else None


def append(data, table, first, counts, k, v, page, dim):
    """Writes tokens k, v (batch, T, heads, D) into `data` (pages, heads, bytes) in place."""
    batch, tokens, heads, _ = k.shape
    for b in range(batch):
        for t in range(tokens if counts is None else min(tokens, int(counts[b]))):
            at = place(table[b], data.shape[0], page, int(first[b]) + t)
            if at is None:
                continue
            ko, vo, kso, vso = token_offsets(page, dim, at[1])
            (kc, ks), (vc, vs) = quantize(k[b, t]), quantize(v[b, t])
            for h in range(heads):
                data[at[0], h, ko] = kc[h].reshape(-1)
                data[at[0], h, vo] = vc[h].reshape(-1)
                data[at[0], h, kso] = ks[h, :dim // BLOCK]
                data[at[0], h, vso] = vs[h, :dim // BLOCK]


def read(data, table_row, page, dim, head, tokens):
    """Keys and values (len(tokens), D) float64 of a head and which of the tokens have a page."""
    keys, values, there = np.zeros((len(tokens), dim)), np.zeros((len(tokens), dim)), np.zeros(len(tokens), bool)
    for i, t in enumerate(tokens):
        at = place(table_row, data.shape[0], page, t)
        if at is None:
            continue
        there[i] = True
        ko, vo, kso, vso = token_offsets(page, dim, at[1])
        row = data[at[0], head]
        keys[i] = dequantize(row[ko].reshape(1, -1, 16), row[kso].reshape(1, -1), dim)[0]
        values[i] = dequantize(row[vo].reshape(1, -1, 16), row[vso].reshape(1, -1), dim)[0]
    return keys, values, there


def attend(q, data, table, lengths, page, scale, window=0, sinks=0):
    """(batch, Lq, Hq, D) -> the result, and for each of its numbers the weighted sum of magnitudes."""
    batch, nq, hq, dim = q.shape
    heads = data.shape[1]
    group = hq // heads
    out, mags = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(batch):
        length = int(np.clip(lengths[b], 0, table.shape[1] * page))
        for h in range(heads):
            keys, values, there = read(data, table[b], page, dim, h, range(length))
            for i in range(nq):
                p = length - nq + i
                t = np.arange(length)
                seen = there & (t <= p) & ((window == 0) | (p - t < window) | (t < sinks))
                if not seen.any():
                    continue
                for g in range(group):
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = keys[seen] @ q[b, i, h * group + g] * scale
                        top = s.max()
                        if top == -np.inf:
                            continue
                        w = np.exp(s - top)
                        w /= w.sum()
                        out[b, i, h * group + g] = w @ values[seen]
                        mags[b, i, h * group + g] = w @ np.abs(values[seen])
    return out, mags
