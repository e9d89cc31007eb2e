"""Sizes for every way in which products and attention on microscaled 4-bit floats are computed: what the library makes of
sizes is asked through `gs_test_mx4_dot_plan` and `gs_test_mx4_attend_plan`, on the host; and attention from its definition in
float64, all rows of a cache head at once, for the sizes that take the other oracle too long."""

import ctypes

import numpy as np

from oracle import mx4
from paper_2105_09377_amd import binding as gs

DIMS = (64, 96, 128, 192, 256)


def mx4_cache(n_pages, heads, page, dim):
    c = gs.gs_mx4_cache()
    c.data, c.n_pages, c.page_size, c.heads, c.head_dim, c.reserved = 0x10000, n_pages, page, heads, dim, 0
    return c


def pattern(shape, n_access, dtype):
    a = gs.gs_ap()
    a.data, a.dtype, a.rank, a.n_access, a.reserved = 0x10000, dtype, len(shape), n_access, 0
    for i, s in enumerate(shape):
        a.shape[i] = s
    return a


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------


def attend_plan(case, window, sinks):
    """(rows, waves, how parts are made) of a case: `whole` sequences, parts `alike` in number, `shares` of one length; `alone`
    where a row's parts have a workgroup to join them."""
    width = -(-case["longest"] // case["page"])
    q = pattern((case["batch"], case["queries"], case["heads"] * case["group"], case["dim"]), 3, gs.GS_BF16)
    table = pattern((case["batch"], width), 1, gs.GS_I32)
    plan = (ctypes.c_int * 5)()
    st = gs.lib().gs_test_mx4_attend_plan(ctypes.byref(q), ctypes.byref(mx4_cache(8, case["heads"], case["page"], case["dim"])),
                                          ctypes.byref(table), ctypes.c_int64(window), ctypes.c_int64(sinks), plan)
    assert st == gs.GS_OK
    rows, waves, parts, slots, alone = plan
    how = "whole" if parts == 1 else ("shares" if slots else "alike") + (" alone" if alone else "")
    return rows, waves, how


def windows(case):
    """Everything, and a window that leaves a few tokens of the longest sequence unseen."""
    return (0, 0), (case["longest"] - 150 if case["longest"] > 400 else 40, 9)


def _attentions():
    for dim in DIMS:
        wide = dim > 128
        some = [  # rows, waves, how: batch, queries, heads, group, page, longest
            ((16, 8, "whole"), 3, 1, 2, 7, 16, 199), ((16, 8, "shares"), 3, 2, 1, 5, 48, 2300), ((16, 8, "shares alone"), 1, 1, 2, 4, 64, 4405),
            ((16, 8, "alike"), 66, 1, 1, 3, 16, 1101),
            ((16, 4, "whole"), 33, 1, 8, 2, 32, 150), ((16, 4, "shares"), 6, 1, 8, 3, 64, 3001), ((16, 4, "shares alone"), 5, 3, 8, 5, 128, 4300),
            ((16, 4, "alike"), 66, 1, 2, 4, 64, 1101),
            ((32, 4, "whole"), 3, 5, 2, 4, 16, 301), ((32, 4, "shares"), 2, 1, 2, 31, 32, 1501), ((32, 4, "shares alone"), 1, 3, 1, 8, 16, 4405),
            ((32, 4, "alike"), 66, 2, 1, 9, 16, 741),
            ((128, 4, "whole"), 3, 40, 2, 1, 16, 199), ((128, 4, "alike"), 2, 150 if wide else 45, 1, 2, 64, 1501), ((128, 4, "alike alone"), 1, 41, 1, 1, 32, 2601)]
        if not wide:
            some += [((16, 4, "alike alone"), 66, 1, 1, 2, 64, 4501), ((256, 8, "whole"), 3, 10, 1, 16, 16, 199), ((256, 8, "alike"), 1, 70, 2, 3, 64, 1301),
                     ((256, 8, "alike alone"), 1, 150, 1, 2, 32, 2601)]
        for way, batch, queries, heads, group, page, longest in some:
            yield {"way": way, "batch": batch, "queries": queries, "heads": heads, "group": group, "dim": dim, "page": page, "longest": longest}


ATTENTIONS = list(_attentions())


def lengths(case):
    """The longest first, then from nothing to it."""
    batch, top = case["batch"], case["longest"]
    n = [top] + [int(top * (b / batch) ** 2) for b in range(1, batch)]
    if batch > 2:
        n[1], n[2] = 0, 1
    return n


def read_head(data, table_row, page, dim, head, length):
    """Keys and values (length, D) float64 of a head and which of the tokens have a page, as mx4.read has them."""
    pages = np.repeat(np.asarray(table_row, dtype=np.int64), page)[:length]
    slots = np.arange(length) % page
    there = (pages >= 0) & (pages < data.shape[0])
    offsets = [np.stack(part) for part in zip(*(mx4.token_offsets(page, dim, s) for s in range(page)))]
    rows = data[np.where(there, pages, 0), head]
    k, v, ks, vs = (np.take_along_axis(rows, part[slots], 1) for part in offsets)
    keys = mx4.dequantize(k.reshape(length, -1, 16), ks, dim)
    values = mx4.dequantize(v.reshape(length, -1, 16), vs, dim)
    return np.where(there[:, None], keys, 0.0), np.where(there[:, None], values, 0.0), there


def attend(q, data, table, lens, page, scale, window=0, sinks=0):
    """mx4.attend, all rows of a cache head at once."""
    batch, nq, hq, dim = q.shape
    heads = data.shape[1]
    group = hq // heads
    out, mags = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(batch):
        length = int(np.clip(lens[b], 0, table.shape[1] * page))
        if length == 0:
            continue
        t, at = np.arange(length), np.repeat(length - nq + np.arange(nq), group)[:, None]
        for h in range(heads):
            keys, values, there = read_head(data, table[b], page, dim, h, length)
            seen = there & (t <= at) & ((window == 0) | (at - t < window) | (t < sinks))
            rows = q[b, :, h * group:(h + 1) * group].reshape(nq * group, dim)
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(seen, rows @ keys.T * scale, -np.inf)
                top = s.max(1, keepdims=True)
                w = np.where(seen, np.exp(s - np.where(top == -np.inf, 0.0, top)), 0.0)
                total = w.sum(1, keepdims=True)
                w /= np.where(total == 0, 1.0, total)
            odd = np.nonzero(~np.isfinite(values).all(1))[0]
            tame = values.copy()
            tame[odd] = 0.0
            o, m = w @ tame, w @ np.abs(tame)
            for i in odd:                                # (a weight of zero is no reason for a row that does not see it)
                o[seen[:, i]] += w[seen[:, i], i, None] * values[i]
                m[seen[:, i]] += w[seen[:, i], i, None] * np.abs(values[i])
            out[b, :, h * group:(h + 1) * group] = o.reshape(nq, group, dim)
            mags[b, :, h * group:(h + 1) * group] = m.reshape(nq, group, dim)
    return out, mags


# ------------------------------------------------------------------------------------------------
# products
# ------------------------------------------------------------------------------------------------

WAYS = ("rows 1", "rows 2", "64x64 few", "64x64", "128x128 few", "128x128 long", "128x128", "256x256",      # as mx4.h counts them
        "weights 32x128", "weights 64x64", "weights 64x128", "weights 128x128", "weights 128x256")


def dot_plan(x_is_bf16, m, n, k):
    """(way, workgroups that share a sum)."""
    plan = (ctypes.c_int * 2)()
    gs.lib().gs_test_mx4_dot_plan(int(x_is_bf16), ctypes.c_int64(m), ctypes.c_int64(n), ctypes.c_int64(k), plan)
    return WAYS[plan[0]], plan[1]


def paired(k):
    """Whether the scales of two slabs of a row come together."""
    return -(-k // 256) * 8 % 16 == 0


# way, scales in pairs: m, n, k
DOTS = {("rows 1", False): (9, 45, 700), ("rows 1", True): (3, 100, 1000), ("rows 2", False): (16, 8200, 600), ("rows 2", True): (33, 1600, 480),
        ("64x64 few", False): (70, 4100, 1200), ("64x64 few", True): (70, 4100, 903), ("64x64", False): (1021, 1500, 601), ("64x64", True): (1021, 1500, 831),
        ("128x128 few", False): (1790, 1800, 561), ("128x128 few", True): (1790, 1800, 1001), ("128x128 long", False): (1700, 1800, 4161),
        ("128x128 long", True): (1700, 1800, 4400), ("128x128", False): (2100, 2200, 601), ("128x128", True): (2100, 2200, 301),
        ("256x256", False): (3500, 3400, 601), ("256x256", True): (3500, 3400, 801)}
# way, shared sums, rows that are padded first: m, n, k
WEIGHT_DOTS = {("rows 1", False, False): (17, 100, 1000), ("rows 2", False, False): (33, 700, 1003),
               ("weights 32x128", False, False): (17, 5000, 264), ("weights 32x128", False, True): (17, 5000, 267),
               ("weights 32x128", True, False): (17, 100, 6200), ("weights 32x128", True, True): (17, 100, 6203),
               ("weights 64x64", False, False): (300, 3250, 264), ("weights 64x64", False, True): (300, 3250, 267),
               ("weights 64x64", True, False): (900, 300, 3000), ("weights 64x64", True, True): (900, 300, 3003),
               ("weights 64x128", False, False): (257, 11000, 264), ("weights 64x128", False, True): (257, 11000, 267),
               ("weights 64x128", True, False): (33, 11000, 5000), ("weights 64x128", True, True): (33, 11000, 5003),
               ("weights 128x128", False, False): (400, 5000, 264), ("weights 128x128", False, True): (400, 5000, 267),
               ("weights 128x128", True, False): (65, 6000, 5000), ("weights 128x128", True, True): (65, 6000, 5003),
               ("weights 128x256", False, False): (400, 11000, 264), ("weights 128x256", False, True): (400, 11000, 267),
               ("weights 128x256", True, False): (65, 11000, 4104), ("weights 128x256", True, True): (65, 11000, 4107)}
