"""What the entry points on scaled 8-bit floats, norms and tokens dealt to experts refuse, without a GPU: nothing is launched by any call
here."""

import ctypes

import pytest
import torch

from paper_2105_09377_amd import binding as gs
from test_abi_host import FAKE, ap

F32, BF, I32 = gs.GS_F32, gs.GS_BF16, gs.GS_I32


def f8(shape, n_access, block_rows=1, values=FAKE, scales=FAKE, reserved=0):
    m = gs.gs_f8()
    m.values, m.scales, m.rank, m.n_access, m.block_rows, m.reserved = values, scales, len(shape), n_access, block_rows, reserved
    for i, s in enumerate(shape):
        m.shape[i] = s
    return m


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_struct_layout():
    assert ctypes.sizeof(gs.gs_f8) == 32 + 8 * gs.GS_MAX_RANK and gs.gs_f8.shape.offset == 32


@pytest.mark.parametrize("m,want", [
    (f8((3, 128), 1), (384, 48)), (f8((3, 129), 1), (768, 48)), (f8((3, 513), 1), (3 * 640, 3 * 32)), (f8((300, 128), 1, 128), (300 * 128, 3 * 16)),
    (f8((2, 130, 4, 100), 2, 128), (2 * 130 * 512, 2 * 2 * 16)), (f8((2, 130, 400), 2), (260 * 512, 260 * 16)), (f8((5, 0), 1), (0, 0)),
    (f8((0, 64), 1, 128), (0, 0)), (f8((257,), 0), (384, 16)), (f8((257,), 0, 128), (384, 16)), (f8((), 0), (128, 16))])
def test_sizes(m, want):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert gs.lib().glenside_f8_sizes(ref(m), ctypes.byref(a), ctypes.byref(b)) == gs.GS_OK
    assert (a.value, b.value) == want


@pytest.mark.parametrize("m,status", [
    (f8((2, 3), 3), gs.GS_ERR_RANK), (f8((2, 3), -1), gs.GS_ERR_RANK), (f8((2, -3), 1), gs.GS_ERR_SHAPE), (f8((1 << 30, 1 << 30), 1), gs.GS_ERR_UNSUPPORTED),
    (f8((1 << 39, 3), 1), gs.GS_ERR_UNSUPPORTED), (f8((1 << 35, 1, 1), 2, 128), gs.GS_ERR_UNSUPPORTED), (f8((0, 1 << 40, 1 << 40), 1), gs.GS_ERR_UNSUPPORTED),
    (f8((2, 3), 1, 64), gs.GS_ERR_UNSUPPORTED), (f8((2, 3), 1, 0), gs.GS_ERR_UNSUPPORTED), (f8((2, 3), 1, reserved=1), gs.GS_ERR_UNSUPPORTED), (None, gs.GS_ERR_NULL)])
def test_impossible_patterns(m, status):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert gs.lib().glenside_f8_sizes(ref(m), ctypes.byref(a), ctypes.byref(b)) == status


@pytest.mark.parametrize("x,m,status", [
    (ap((4, 64), 1), f8((4, 64), 1, values=None), gs.GS_ERR_NULL), (ap((4, 64), 1), f8((4, 64), 1, scales=None), gs.GS_ERR_NULL),
    (ap((4, 64), 1), f8((4, 64), 1, values=FAKE + 8), gs.GS_ERR_UNSUPPORTED), (ap((4, 64), 1), f8((4, 64), 1, scales=FAKE + 4), gs.GS_ERR_UNSUPPORTED),
    (ap((4, 64), 1, data=FAKE + 2), f8((4, 64), 1), gs.GS_ERR_UNSUPPORTED), (ap((4, 64), 1, data=None), f8((4, 64), 1), gs.GS_ERR_NULL),
    (ap((4, 64), 1), f8((4, 64), 2), gs.GS_ERR_RANK), (ap((4, 64), 1), f8((4, 8, 8), 1), gs.GS_ERR_RANK), (ap((4, 64), 1), f8((4, 65), 1, 128), gs.GS_ERR_SHAPE),
    (ap((4, 64), 1, gs.GS_I8), f8((4, 64), 1), gs.GS_ERR_DTYPE), (ap((4, 64), 1, gs.GS_F8), f8((4, 64), 1), gs.GS_ERR_DTYPE),
    (ap((4, 64), 1), f8((4, 64), 1, 2), gs.GS_ERR_UNSUPPORTED), (None, f8((4, 64), 1), gs.GS_ERR_NULL), (ap((4, 64), 1), None, gs.GS_ERR_NULL)])
def test_conversions_refuse(x, m, status):
    L = gs.lib()
    assert L.glenside_f8_quantize(ref(x), ref(m), None) == status
    assert L.glenside_f8_dequantize(ref(m), ref(x), None) == status


def norm(**kw):
    a = dict(x=ap((4, 64), 1), residual=ap((4, 64), 1), weight=ap((64,), 0), eps=1e-6, total=ap((4, 64), 1), out=ap((4, 64), 1, F32), codes=f8((4, 64), 1))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), gs.GS_ERR_NULL), (dict(x=ap((4, 64), 1, I32)), gs.GS_ERR_DTYPE), (dict(x=ap((4, 64), 1, data=FAKE + 2)), gs.GS_ERR_UNSUPPORTED),
    (dict(residual=ap((4, 64), 1, F32)), gs.GS_ERR_DTYPE), (dict(residual=ap((3, 64), 1)), gs.GS_ERR_SHAPE), (dict(residual=ap((4, 64), 2)), gs.GS_ERR_RANK),
    (dict(total=ap((4, 64), 1, F32)), gs.GS_ERR_DTYPE), (dict(total=ap((4, 65), 1)), gs.GS_ERR_SHAPE), (dict(total=ap((4, 64), 1, data=None)), gs.GS_ERR_NULL),
    (dict(weight=ap((63,), 0)), gs.GS_ERR_SHAPE), (dict(weight=ap((64,), 1)), gs.GS_ERR_RANK), (dict(weight=ap((8, 8), 0)), gs.GS_ERR_RANK),
    (dict(weight=ap((64,), 0, gs.GS_I8)), gs.GS_ERR_DTYPE), (dict(eps=-1e-6), gs.GS_ERR_UNSUPPORTED), (dict(eps=float("nan")), gs.GS_ERR_UNSUPPORTED),
    (dict(eps=float("inf")), gs.GS_ERR_UNSUPPORTED), (dict(out=None, codes=None), gs.GS_ERR_NULL),
    (dict(out=ap((4, 8, 8), 1), codes=f8((4, 8, 8), 1)), gs.GS_ERR_RANK), (dict(out=ap((4, 63), 1), codes=f8((4, 63), 1)), gs.GS_ERR_SHAPE)])
def test_norms_refuse(kw, status):
    L, a = gs.lib(), norm(**kw)
    args = [ref(a["x"]), ref(a["residual"]), ref(a["weight"]), a["eps"], ref(a["total"])]
    assert L.glenside_norm(*args, ref(a["out"]), None) == status
    assert L.glenside_f8_norm(*args, ref(a["codes"]), None) == status


def test_norms_refuse_their_results():
    L, a = gs.lib(), norm()
    args = [ref(a["x"]), None, None, 1e-6, None]
    assert L.glenside_norm(*args, ref(ap((4, 64), 1, gs.GS_F8)), None) == gs.GS_ERR_DTYPE
    assert L.glenside_f8_norm(*args, ref(f8((4, 64), 1, 128)), None) == gs.GS_ERR_UNSUPPORTED


@pytest.mark.parametrize("a0,a1,out,act,status", [
    (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6), 2, I32), 0, gs.GS_ERR_DTYPE), (f8((4, 64), 1), f8((6, 32), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_SHAPE),
    (f8((4, 2, 32), 1), f8((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_SHAPE), (f8((4, 64), 1), f8((6, 64), 1, 128), ap((6, 4), 2, F32), 0, gs.GS_ERR_SHAPE),
    (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6), 1, F32), 0, gs.GS_ERR_RANK), (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6, 1), 3, F32), 0, gs.GS_ERR_RANK),
    (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6), 2, F32), 7, gs.GS_ERR_UNSUPPORTED), (f8((4, 64), 1, values=None), f8((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL),
    (f8((4, 64), 1), f8((6, 64), 1, scales=None), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL), (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6), 2, F32, data=None), 0, gs.GS_ERR_NULL),
    (f8((4, 64), 1), f8((6, 64), 1), ap((4, 6), 2, F32, data=FAKE + 4), 0, gs.GS_ERR_UNSUPPORTED), (None, f8((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL),
    (f8((4, 64), 1), None, ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL), (f8((4, 64), 1), f8((6, 64), 1), None, 0, gs.GS_ERR_NULL),
    (f8((4, 64), 1), f8((2, 6, 64), 2, 128), ap((4, 2, 6), 3, F32), 0, gs.GS_ERR_UNSUPPORTED),
    (f8((2, 6, 64), 2, 128), f8((4, 64), 1), ap((2, 6, 4), 3, F32), 0, gs.GS_ERR_UNSUPPORTED)])
def test_products_refuse(a0, a1, out, act, status):
    assert gs.lib().glenside_f8_dot(ref(a0), ref(a1), ref(out), act, None, 0, None) == status


def test_products_want_their_workspace():
    L = gs.lib()
    a0, a1, out = f8((64, 8192), 1), f8((8192, 8192), 1, 128), ap((64, 8192), 2, F32)
    need = L.glenside_f8_dot_workspace(ref(a0), ref(a1))
    assert need > 0 and need % (4 * 64 * 8192) == 0
    for ws, n in ((None, 0), (FAKE, need - 1), (FAKE + 4, need)):
        assert L.glenside_f8_dot(ref(a0), ref(a1), ref(out), 0, ws, n, None) == gs.GS_ERR_WORKSPACE
    assert L.glenside_f8_dot_workspace(ref(f8((1, 8192), 1)), ref(a1)) == 0
    assert L.glenside_f8_dot_workspace(ref(f8((64, 8191), 1)), ref(a1)) == 0
    assert L.glenside_f8_dot_workspace(None, ref(a1)) == 0
    assert L.glenside_f8_expert_dot_workspace(ref(a0), 64, ref(f8((4, 128, 8192), 2, 128))) == 0
    assert L.glenside_f8_expert_dot_workspace(ref(a0), 64, ref(f8((0, 8192, 8192), 2, 128))) == 0
    assert L.glenside_f8_expert_dot_workspace(ref(a0), -1, ref(f8((4, 128, 8192), 2, 128))) == 0


def experts_dot(**kw):
    a = dict(a0=f8((10, 64), 1), tokens=ap((30,), 1, I32), offsets=ap((5,), 1, I32), w=f8((4, 6, 64), 2, 128), out=ap((30, 6), 2, F32), act=0)
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(a0=None), gs.GS_ERR_NULL), (dict(w=None), gs.GS_ERR_NULL), (dict(offsets=None), gs.GS_ERR_NULL), (dict(out=None), gs.GS_ERR_NULL),
    (dict(w=f8((24, 64), 1, 128)), gs.GS_ERR_RANK), (dict(w=f8((2, 2, 6, 64), 3, 128)), gs.GS_ERR_RANK), (dict(w=f8((4, 6, 65), 2, 128)), gs.GS_ERR_SHAPE),
    (dict(offsets=ap((4,), 1, I32)), gs.GS_ERR_SHAPE), (dict(offsets=ap((5,), 1, F32)), gs.GS_ERR_DTYPE), (dict(offsets=ap((5, 1), 2, I32)), gs.GS_ERR_RANK),
    (dict(tokens=ap((29,), 1, I32)), gs.GS_ERR_SHAPE), (dict(tokens=ap((30,), 1, BF)), gs.GS_ERR_DTYPE), (dict(tokens=ap((30,), 0, I32)), gs.GS_ERR_RANK),
    (dict(tokens=None), gs.GS_ERR_SHAPE), (dict(out=ap((30, 7), 2, F32)), gs.GS_ERR_SHAPE), (dict(out=ap((30, 6, 1), 3, F32)), gs.GS_ERR_RANK),
    (dict(out=ap((30, 6), 1, F32)), gs.GS_ERR_RANK), (dict(out=ap((30, 6), 2, I32)), gs.GS_ERR_DTYPE), (dict(act=2), gs.GS_ERR_UNSUPPORTED),
    (dict(a0=f8((2, 5, 64), 2, 128)), gs.GS_ERR_UNSUPPORTED), (dict(w=f8((4, 6, 64), 2, 128, values=FAKE + 1)), gs.GS_ERR_UNSUPPORTED)])
def test_experts_products_refuse(kw, status):
    a = experts_dot(**kw)
    assert gs.lib().glenside_f8_expert_dot(ref(a["a0"]), ref(a["tokens"]), ref(a["offsets"]), ref(a["w"]), ref(a["out"]), a["act"], None, 0, None) == status


def test_no_experts_launch_nothing():
    """Not even where as many rows of one matrix would share sums in a workspace."""
    a = experts_dot(a0=f8((64, 8192), 1), w=f8((0, 8192, 8192), 2, 128), offsets=ap((1,), 1, I32), tokens=None, out=ap((64, 8192), 2, F32))
    assert gs.lib().glenside_f8_expert_dot(ref(a["a0"]), None, ref(a["offsets"]), ref(a["w"]), ref(a["out"]), 0, None, 0, None) == gs.GS_OK


def sort(**kw):
    a = dict(experts=ap((10, 3), 2, I32), offsets=ap((9,), 1, I32), tokens=ap((30,), 1, I32), places=ap((10, 3), 2, I32))
    a.update(kw)
    return [ref(a[n]) for n in ("experts", "offsets", "tokens", "places")]


@pytest.mark.parametrize("kw,status", [
    (dict(experts=None), gs.GS_ERR_NULL), (dict(experts=ap((10, 3), 1, I32)), gs.GS_ERR_RANK), (dict(experts=ap((30,), 1, I32)), gs.GS_ERR_RANK),
    (dict(experts=ap((10, 3), 2, F32)), gs.GS_ERR_DTYPE), (dict(offsets=ap((0,), 1, I32)), gs.GS_ERR_SHAPE), (dict(offsets=ap((4098,), 1, I32)), gs.GS_ERR_UNSUPPORTED),
    (dict(tokens=ap((29,), 1, I32)), gs.GS_ERR_SHAPE), (dict(places=ap((3, 10), 2, I32)), gs.GS_ERR_SHAPE), (dict(places=None), gs.GS_ERR_NULL),
    (dict(places=ap((10, 3), 2, I32, data=FAKE + 4)), gs.GS_ERR_UNSUPPORTED),
    (dict(experts=ap((1 << 20, 1 << 11), 2, I32), tokens=ap((1 << 31,), 1, I32), places=ap((1 << 20, 1 << 11), 2, I32)), gs.GS_ERR_UNSUPPORTED)])
def test_sorting_refuses(kw, status):
    assert gs.lib().glenside_expert_sort(*sort(**kw), None, 0, None) == status


def test_sorting_wants_its_workspace():
    L = gs.lib()
    need = L.glenside_expert_sort_workspace(60000, 64)
    many = dict(experts=ap((20000, 3), 2, I32), offsets=ap((65,), 1, I32), tokens=ap((60000,), 1, I32), places=ap((20000, 3), 2, I32))
    assert need > 0
    for ws, n in ((None, 0), (FAKE, need - 1), (FAKE + 8, need)):
        assert L.glenside_expert_sort(*sort(**many), ws, n, None) == gs.GS_ERR_WORKSPACE
    assert L.glenside_expert_sort_workspace(500, 64) == 0
    for bad in ((-1, 4), (4, -1), (4, 4097), (1 << 31, 4)):
        assert L.glenside_expert_sort_workspace(*bad) == 0


def rows(**kw):
    a = dict(flat=ap((10, 5, 8), 1), rows=ap((30, 5, 8), 1), places=ap((10, 3), 2, I32), weights=ap((10, 3), 2, F32), grad_rows=ap((30, 5, 8), 1), grad_weights=ap((10, 3), 2, F32))
    a.update(kw)
    return {n: ref(v) for n, v in a.items()}


@pytest.mark.parametrize("kw,status", [
    (dict(flat=None), gs.GS_ERR_NULL), (dict(rows=None), gs.GS_ERR_NULL), (dict(places=None), gs.GS_ERR_NULL), (dict(flat=ap((9, 5, 8), 1)), gs.GS_ERR_SHAPE),
    (dict(flat=ap((10, 40), 1)), gs.GS_ERR_RANK), (dict(flat=ap((10, 5, 8), 2)), gs.GS_ERR_RANK), (dict(rows=ap((30, 5, 9), 1)), gs.GS_ERR_SHAPE),
    (dict(rows=ap((30, 5, 8), 0)), gs.GS_ERR_RANK), (dict(places=ap((10, 3), 2, F32)), gs.GS_ERR_DTYPE), (dict(places=ap((30,), 1, I32)), gs.GS_ERR_RANK),
    (dict(rows=ap((30, 5, 8), 1, data=FAKE + 2)), gs.GS_ERR_UNSUPPORTED)])
def test_rows_refuse(kw, status):
    L, a = gs.lib(), rows(**kw)
    assert L.glenside_expert_split(a["flat"], a["places"], a["rows"], None) == status
    assert L.glenside_expert_join(a["rows"], a["places"], a["weights"], a["flat"], None) == status
    assert L.glenside_expert_join_grad(a["flat"], a["rows"], a["places"], a["weights"], a["grad_rows"], a["grad_weights"], None) == status


def test_rows_refuse_types_and_weights():
    L = gs.lib()
    a = rows(flat=ap((10, 5, 8), 1, F32))
    assert L.glenside_expert_split(a["flat"], a["places"], a["rows"], None) == gs.GS_ERR_DTYPE
    assert L.glenside_expert_join_grad(a["flat"], a["rows"], a["places"], None, a["grad_rows"], None, None) == gs.GS_ERR_DTYPE
    a = rows(flat=ap((10, 5, 8), 1, gs.GS_I8), rows=ap((30, 5, 8), 1, gs.GS_I8))
    assert L.glenside_expert_join(a["rows"], a["places"], a["weights"], a["flat"], None) == gs.GS_ERR_DTYPE
    for weights, status in ((ap((10, 4), 2, F32), gs.GS_ERR_SHAPE), (ap((10, 3), 2, BF), gs.GS_ERR_DTYPE), (ap((10, 3), 1, F32), gs.GS_ERR_RANK)):
        a = rows(weights=weights, grad_weights=weights)
        assert L.glenside_expert_join(a["rows"], a["places"], a["weights"], a["flat"], None) == status
        assert L.glenside_expert_join_grad(a["flat"], a["rows"], a["places"], None, a["grad_rows"], a["grad_weights"], None) == status
    for bad, status in ((ap((29, 5, 8), 1), gs.GS_ERR_SHAPE), (ap((30, 5, 8), 1, F32), gs.GS_ERR_DTYPE), (None, gs.GS_ERR_NULL)):
        a = rows(grad_rows=bad)
        assert L.glenside_expert_join_grad(a["flat"], a["rows"], a["places"], a["weights"], a["grad_rows"], a["grad_weights"], None) == status


def at(place, shape, n_access, dtype=BF):
    """A pattern in a megabyte of its own."""
    return ap(shape, n_access, dtype, data=FAKE + place * (1 << 20))


def test_nothing_works_in_place():
    """A result that shares bytes with an input, from its first or only its last, is refused; norms of long rows read their inputs twice."""
    L, no = gs.lib(), gs.GS_ERR_UNSUPPORTED
    x, residual, weight, total, out = at(1, (4, 64), 1), at(2, (4, 64), 1), at(3, (64,), 0), at(4, (4, 64), 1), at(5, (4, 64), 1)
    codes = f8((4, 64), 1, values=FAKE + (9 << 20), scales=FAKE + (10 << 20))
    for of in (x, residual, weight):
        for back in (0, 4 * 64 * 2 - 16):
            onto = ap((4, 64), 1, data=of.data - back)
            args = [ref(x), ref(residual), ref(weight), 1e-6]
            assert L.glenside_norm(*args, ref(onto), ref(out), None) == no
            assert L.glenside_norm(*args, ref(total), ref(onto), None) == no
            assert L.glenside_f8_norm(*args, ref(onto), ref(codes), None) == no
    experts, offsets = at(1, (10, 3), 2, I32), at(2, (5,), 1, I32)
    tokens, places = at(3, (30,), 1, I32), at(4, (10, 3), 2, I32)
    for three in ((ap((5,), 1, I32, data=experts.data), tokens, places), (offsets, ap((30,), 1, I32, data=experts.data), places),
                  (offsets, tokens, ap((10, 3), 2, I32, data=experts.data - 112))):
        assert L.glenside_expert_sort(ref(experts), *(ref(t) for t in three), None, 0, None) == no
    flat, rows_, weights = at(1, (10, 40), 1), at(2, (30, 40), 1), at(5, (10, 3), 2, F32)
    grad_rows, grad_weights = at(6, (30, 40), 1), at(7, (10, 3), 2, F32)
    for of in (flat, places):
        assert L.glenside_expert_split(ref(flat), ref(places), ref(ap((30, 40), 1, data=of.data)), None) == no
    for of in (rows_, places, weights):
        assert L.glenside_expert_join(ref(rows_), ref(places), ref(weights), ref(ap((10, 40), 1, data=of.data)), None) == no
    for of in (flat, rows_, places, weights):
        args = [ref(flat), ref(rows_), ref(places), ref(weights)]
        assert L.glenside_expert_join_grad(*args, ref(ap((30, 40), 1, data=of.data)), ref(grad_weights), None) == no
        assert L.glenside_expert_join_grad(*args, ref(grad_rows), ref(ap((10, 3), 2, F32, data=of.data)), None) == no


def refused(status, call, *args, **kw):
    with pytest.raises(gs.GlensideError) as e:
        call(*args, **kw)
    assert e.value.status == status


def test_binding_refuses():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    m = gs.F8(torch.zeros(4, 1, 128, dtype=torch.uint8), torch.zeros(4, 4), (4, 64), 1)
    refused(gs.GS_ERR_DTYPE, gs.f8_quantize, x.to(torch.int8))
    refused(gs.GS_ERR_RANK, gs.f8_quantize, x, 3)
    refused(gs.GS_ERR_UNSUPPORTED, gs.f8_quantize, x, block_rows=32)
    refused(gs.GS_ERR_SHAPE, gs.f8_quantize, x, out=m._replace(shape=(4, 65)))
    refused(gs.GS_ERR_SHAPE, gs.f8_dequantize, m._replace(shape=(4, 129)))          # more blocks than there are
    refused(gs.GS_ERR_SHAPE, gs.f8_dequantize, m._replace(scales=torch.zeros(3, 4)))
    refused(gs.GS_ERR_RANK, gs.f8_dequantize, m._replace(n_access=3))
    refused(gs.GS_ERR_UNSUPPORTED, gs.f8_dequantize, m._replace(block_rows=2))
    refused(gs.GS_ERR_DTYPE, gs.f8_dequantize, m, out_dtype=torch.int32)
    refused(gs.GS_ERR_SHAPE, gs.f8_dot, m, m, out=torch.zeros(4, 5))
    refused(gs.GS_ERR_RANK, gs.f8_expert_dot, m, m, torch.zeros(5, dtype=torch.int32))
    refused(gs.GS_ERR_SHAPE, gs.norm, x, torch.zeros(63))
    refused(gs.GS_ERR_UNSUPPORTED, gs.f8_norm, x, eps=-1.0)
    refused(gs.GS_ERR_DTYPE, gs.norm, x, residual=x.float())
    for wrong in (m._replace(scales=torch.zeros(4, 4, dtype=torch.uint8)), m._replace(values=torch.zeros(4, 1, 128)), m._replace(values=torch.zeros(4, 1, 256, dtype=torch.uint8)[:, :, ::2])):
        with pytest.raises(ValueError):
            gs.f8_dequantize(wrong)
    with pytest.raises(ValueError):
        gs.f8_quantize(x.t())
    with pytest.raises(ValueError):
        gs.f8_dot(m, m._replace(values=torch.zeros(4, 1, 128, dtype=torch.uint8, device="meta")))
    with pytest.raises(ValueError):
        gs.norm(x, torch.zeros(64, device="meta"))
    for wrong in (x, (1, 2), None, "m"):
        with pytest.raises((TypeError, AttributeError)):
            gs.f8_dequantize(wrong)
    with pytest.raises(TypeError):
        gs.f8_dot(m, m, act=1.0)
    with pytest.raises(TypeError):
        gs.norm(x, eps="1")


def test_binding_refuses_experts():
    e = torch.zeros(4, 2, dtype=torch.int32)
    x, r = torch.zeros(4, 8), torch.zeros(8, 8)
    refused(gs.GS_ERR_DTYPE, gs.expert_sort, e.float(), 4)
    refused(gs.GS_ERR_SHAPE, gs.expert_sort, e, -1)
    refused(gs.GS_ERR_UNSUPPORTED, gs.expert_sort, e, 5000)
    refused(gs.GS_ERR_UNSUPPORTED, gs.expert_sort, e, 1 << 40)
    refused(gs.GS_ERR_RANK, gs.expert_sort, e[0].contiguous(), 4)
    three = gs.ExpertSort(torch.zeros(5, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), e.clone())
    refused(gs.GS_ERR_SHAPE, gs.expert_sort, e, 3, out=three)
    refused(gs.GS_ERR_SHAPE, gs.expert_split, x[:3].contiguous(), e)
    refused(gs.GS_ERR_DTYPE, gs.expert_split, x, e, out=r.to(torch.bfloat16))
    refused(gs.GS_ERR_SHAPE, gs.expert_join, r, e, torch.zeros(4, 3))
    refused(gs.GS_ERR_DTYPE, gs.expert_join, r, e.float())
    refused(gs.GS_ERR_DTYPE, gs.expert_join_grad, x, r.to(torch.bfloat16), e)
    refused(gs.GS_ERR_SHAPE, gs.expert_join_grad, x, r, e, grad_weights=torch.zeros(4, 3))
    with pytest.raises(ValueError):
        gs.expert_split(x.t(), e)
    with pytest.raises(ValueError):
        gs.expert_join(r, e.to("meta"))
    with pytest.raises(ValueError):
        gs.expert_split(torch.zeros(()), e)
    with pytest.raises(TypeError):
        gs.expert_sort(e, 4, out=(1, 2))
