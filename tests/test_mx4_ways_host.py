"""Every way in which products and attention on microscaled 4-bit floats are computed has a test that takes it: if a rule changes, the
sizes in mx4_ways.py change with it.  Without a GPU."""

import numpy as np
import pytest

import mx4_ways
from oracle import mx4


@pytest.mark.parametrize("case", mx4_ways.ATTENTIONS, ids=lambda c: "{way}-{dim}".format(**c))
def test_attentions_go_where_they_are_meant_to(case):
    for window, sinks in mx4_ways.windows(case):
        assert mx4_ways.attend_plan(case, window, sinks) == case["way"]


def test_attentions_take_every_way():
    """Each kernel that the library is built with, and each way of making parts that it can be asked for."""
    for dim in mx4_ways.DIMS:
        # 16 rows, alike, alone: 65 sequences and more in parts of nine and more, which are more than the chip has room for in wide heads
        rows = {(16, 8): ("whole", "shares", "shares alone", "alike"), (32, 4): ("whole", "shares", "shares alone", "alike"),
                (16, 4): ("whole", "shares", "shares alone", "alike") + (("alike alone",) if dim <= 128 else ()),
                (128, 4): ("whole", "alike", "alike alone")}
        if dim <= 128:
            rows[256, 8] = ("whole", "alike", "alike alone")
        want = {(*shape, how) for shape, hows in rows.items() for how in hows}
        assert {c["way"] for c in mx4_ways.ATTENTIONS if c["dim"] == dim} == want


def test_attentions_of_other_sizes_take_no_other_way():
    ways = {(c["dim"], c["way"]) for c in mx4_ways.ATTENTIONS}
    for dim in mx4_ways.DIMS:
        for batch in (1, 2, 5, 16, 33, 64, 65, 130, 300, 1000):
            for heads in (1, 2, 8, 40):
                for queries, group in ((1, 1), (1, 16), (1, 17), (4, 8), (40, 1), (129, 1), (500, 4), (9, 64)):
                    for longest in (1, 200, 513, 1030, 5000, 70000):
                        case = {"batch": batch, "queries": queries, "heads": heads, "group": group, "dim": dim, "page": 64, "longest": longest}
                        for window in (0, 100, 4096):
                            assert (dim, mx4_ways.attend_plan(case, window, 4)) in ways, case


@pytest.mark.parametrize("key", mx4_ways.DOTS, ids=str)
def test_products_go_where_they_are_meant_to(key):
    m, n, k = mx4_ways.DOTS[key]
    assert mx4_ways.dot_plan(False, m, n, k) == (key[0], 1) and mx4_ways.paired(k) == key[1]


@pytest.mark.parametrize("key", mx4_ways.WEIGHT_DOTS, ids=str)
def test_products_of_weights_go_where_they_are_meant_to(key):
    m, n, k = mx4_ways.WEIGHT_DOTS[key]
    way, splits = mx4_ways.dot_plan(True, m, n, k)
    assert (way, splits > 1) == key[:2] and (k % 8 != 0 and not way.startswith("rows")) == key[2]


def test_products_take_every_way():
    assert {key[0] for key in mx4_ways.DOTS} == set(mx4_ways.WAYS[:8]) and len(mx4_ways.DOTS) == 16
    assert {key[0] for key in mx4_ways.WEIGHT_DOTS} == set(mx4_ways.WAYS[:2] + mx4_ways.WAYS[8:]) and len(mx4_ways.WEIGHT_DOTS) == 22


@pytest.mark.parametrize("dim,page", [(64, 16), (96, 48), (256, 32)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 3)])
def test_attention_at_once_is_attention_row_by_row(dim, page, window, sinks):
    """The float64 values of the large cases against the oracle's, on random bytes: NaN scales, tokens without a page, rows that see nothing."""
    rng = np.random.default_rng(dim + window)
    data = rng.integers(0, 256, (7, 2, mx4.block_bytes(page, dim)), dtype=np.uint8)
    scales = data[:, :, page * dim:]                                        # between 2^-7 and 2^8, a few NaN among those of the values
    scales[...] = 120 + scales % 16
    scales[3, :, scales.shape[2] // 2 + 5] = 255
    table = np.array([[0, 3, 1], [2, -1, 4], [5, 6, 7]])
    q = rng.normal(size=(3, 4, 6, dim)) * 0.01
    lens = [3 * page, 2 * page + 5, 2]
    want, want_mag = mx4.attend(q, data, table, lens, page, 0.1, window, sinks)
    got, mag = mx4_ways.attend(q, data, table, lens, page, 0.1, window, sinks)
    nan = np.isnan(want)
    assert nan.any() == np.isnan(got).any() and np.array_equal(np.isnan(got), nan) and not nan.all()
    # (1e-12: sums of at most 144 products of 64 bits each, in another order, scores below 2^12)
    assert np.allclose(got, want, rtol=0, atol=1e-12 * np.nanmax(want_mag), equal_nan=True)
    assert np.allclose(mag, want_mag, rtol=1e-11, atol=0, equal_nan=True)


def test_heads_are_read_as_the_oracle_reads_them():
    rng = np.random.default_rng(3)
    data = rng.integers(0, 255, (5, 2, mx4.block_bytes(32, 96)), dtype=np.uint8)
    table = np.array([4, -2, 0, 5])
    want = mx4.read(data, table, 32, 96, 1, range(117))
    got = mx4_ways.read_head(data, table, 32, 96, 1, 117)
    for a, b in zip(got, want):
        assert np.array_equal(a, b, equal_nan=True)
