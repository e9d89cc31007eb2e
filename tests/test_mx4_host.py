"""What the entry points on microscaled 4-bit floats refuse, without a GPU: nothing is launched by any call here."""

import ctypes

import pytest
import torch

from paper_2105_09377_amd import binding as gs
from test_abi_host import FAKE, ap


def mx(shape, n_access, values=FAKE, scales=FAKE):
    m = gs.gs_mx4()
    m.values, m.scales, m.rank, m.n_access = values, scales, len(shape), n_access
    for i, s in enumerate(shape):
        m.shape[i] = s
    return m


def cache(pages=8, page=64, heads=2, dim=128, data=FAKE, reserved=0):
    c = gs.gs_mx4_cache()
    c.data, c.n_pages, c.page_size, c.heads, c.head_dim, c.reserved = data, pages, page, heads, dim, reserved
    return c


def ref(x):
    return None if x is None else ctypes.byref(x)


I32 = gs.GS_I32


def test_struct_layouts():
    assert ctypes.sizeof(gs.gs_mx4) == 24 + 8 * gs.GS_MAX_RANK and gs.gs_mx4.shape.offset == 24
    assert ctypes.sizeof(gs.gs_mx4_cache) == 32


@pytest.mark.parametrize("shape,n,want", [((3, 64), 1, (96, 24)), ((3, 65), 1, (144, 24)), ((2, 3, 4, 100), 2, (6 * 13 * 16, 6 * 16)),
                                          ((5, 0), 1, (0, 0)), ((0, 64), 1, (0, 0)), ((257,), 0, (144, 16)), ((), 0, (16, 8))])
def test_sizes(shape, n, want):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert gs.lib().glenside_mx4_sizes(ref(mx(shape, n)), ctypes.byref(a), ctypes.byref(b)) == gs.GS_OK
    assert (a.value, b.value) == want


@pytest.mark.parametrize("m,status", [(mx((2, 3), 3), gs.GS_ERR_RANK), (mx((2, 3), -1), gs.GS_ERR_RANK), (mx((2, -3), 1), gs.GS_ERR_SHAPE),
                                      (mx((1 << 30, 1 << 30), 1), gs.GS_ERR_UNSUPPORTED), (mx((1 << 39, 3), 1), gs.GS_ERR_UNSUPPORTED),
                                      (mx((0, 1 << 40, 1 << 40), 1), gs.GS_ERR_UNSUPPORTED), (None, gs.GS_ERR_NULL)])
def test_impossible_patterns(m, status):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert gs.lib().glenside_mx4_sizes(ref(m), ctypes.byref(a), ctypes.byref(b)) == status


@pytest.mark.parametrize("x,m,status", [
    (ap((4, 64), 1), mx((4, 64), 1, values=None), gs.GS_ERR_NULL),
    (ap((4, 64), 1), mx((4, 64), 1, scales=None), gs.GS_ERR_NULL),
    (ap((4, 64), 1), mx((4, 64), 1, values=FAKE + 8), gs.GS_ERR_UNSUPPORTED),
    (ap((4, 64), 1), mx((4, 64), 1, scales=FAKE + 4), gs.GS_ERR_UNSUPPORTED),
    (ap((4, 64), 1, data=FAKE + 2), mx((4, 64), 1), gs.GS_ERR_UNSUPPORTED),
    (ap((4, 64), 1, data=None), mx((4, 64), 1), gs.GS_ERR_NULL),
    (ap((4, 64), 1), mx((4, 64), 2), gs.GS_ERR_RANK),
    (ap((4, 64), 1), mx((4, 8, 8), 1), gs.GS_ERR_RANK),
    (ap((4, 64), 1), mx((4, 65), 1), gs.GS_ERR_SHAPE),
    (ap((4, 64), 1, gs.GS_I8), mx((4, 64), 1), gs.GS_ERR_DTYPE),
    (ap((4, 64), 1, gs.GS_F8), mx((4, 64), 1), gs.GS_ERR_DTYPE),
    (None, mx((4, 64), 1), gs.GS_ERR_NULL), (ap((4, 64), 1), None, gs.GS_ERR_NULL),
])
def test_conversions_refuse(x, m, status):
    L = gs.lib()
    assert L.glenside_mx4_quantize(ref(x), ref(m), None) == status
    assert L.glenside_mx4_dequantize(ref(m), ref(x), None) == status


F32 = gs.GS_F32


@pytest.mark.parametrize("a0,a1,out,act,status", [
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6), 2, gs.GS_I32), 0, gs.GS_ERR_DTYPE),
    (mx((4, 64), 1), mx((6, 32), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_SHAPE),
    (mx((4, 2, 32), 1), mx((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_SHAPE),
    (mx((4, 64), 1), mx((6, 64), 1), ap((6, 4), 2, F32), 0, gs.GS_ERR_SHAPE),
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6), 1, F32), 0, gs.GS_ERR_RANK),
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6, 1), 3, F32), 0, gs.GS_ERR_RANK),
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6), 2, F32), 7, gs.GS_ERR_UNSUPPORTED),
    (mx((4, 64), 1, values=None), mx((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL),
    (mx((4, 64), 1), mx((6, 64), 1, scales=None), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL),
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6), 2, F32, data=None), 0, gs.GS_ERR_NULL),
    (mx((4, 64), 1), mx((6, 64), 1), ap((4, 6), 2, F32, data=FAKE + 4), 0, gs.GS_ERR_UNSUPPORTED),
    (None, mx((6, 64), 1), ap((4, 6), 2, F32), 0, gs.GS_ERR_NULL),
])
def test_products_refuse(a0, a1, out, act, status):
    L = gs.lib()
    assert L.glenside_mx4_dot(ref(a0), ref(a1), ref(out), act, None, 0, None) == status
    x = None if a0 is None else ap(tuple(a0.shape[i] for i in range(a0.rank)), a0.n_access, data=a0.values)
    assert L.glenside_mx4_weight_dot(ref(x), ref(a1), ref(out), act, None, 0, None) == status


def test_weight_products_take_bfloat16_only():
    for dt in (gs.GS_F32, gs.GS_I8, gs.GS_F8):
        assert gs.lib().glenside_mx4_weight_dot(ref(ap((4, 64), 1, dt)), ref(mx((6, 64), 1)), ref(ap((4, 6), 2, F32)), 0, None, 0, None) == gs.GS_ERR_DTYPE


@pytest.mark.parametrize("c,want", [(cache(), 8 * 2 * (64 * 128 + 2 * 64 * 4)), (cache(page=24), 0), (cache(page=0), 0), (cache(page=4112), 0),
                                    (cache(dim=80), 0), (cache(dim=32), 0), (cache(heads=0), 0), (cache(pages=-1), 0), (cache(reserved=1), 0),
                                    (cache(page=48, dim=96, heads=1, pages=1), 48 * 96 + 2 * 48 * 3), (cache(pages=1 << 40), 0), (None, 0)])
def test_cache_bytes(c, want):
    assert gs.lib().glenside_mx4_cache_bytes(ref(c)) == want


def tokens(**kw):
    a = dict(cache=cache(), table=ap((3, 5), 1, I32), first=ap((3,), 1, I32), counts=None, k=ap((3, 7, 2, 128), 3), v=ap((3, 7, 2, 128), 3))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(cache=cache(page=20)), gs.GS_ERR_UNSUPPORTED), (dict(cache=cache(data=None)), gs.GS_ERR_NULL), (dict(cache=None), gs.GS_ERR_NULL),
    (dict(cache=cache(data=FAKE + 8)), gs.GS_ERR_UNSUPPORTED), (dict(cache=cache(heads=4)), gs.GS_ERR_SHAPE), (dict(cache=cache(dim=64)), gs.GS_ERR_SHAPE),
    (dict(table=ap((3, 5), 1, gs.GS_F32)), gs.GS_ERR_DTYPE), (dict(table=ap((2, 5), 1, I32)), gs.GS_ERR_SHAPE), (dict(table=ap((3, 5), 2, I32)), gs.GS_ERR_RANK),
    (dict(table=ap((3, 1 << 25), 1, I32)), gs.GS_ERR_UNSUPPORTED), (dict(table=ap((3, 5), 1, I32, data=None)), gs.GS_ERR_NULL),
    (dict(first=ap((4,), 1, I32)), gs.GS_ERR_SHAPE), (dict(first=ap((3,), 1, gs.GS_F32)), gs.GS_ERR_DTYPE), (dict(first=ap((3, 1), 1, I32)), gs.GS_ERR_RANK),
    (dict(first=None), gs.GS_ERR_NULL),
    (dict(k=ap((3, 7, 2, 128), 3, gs.GS_F32)), gs.GS_ERR_DTYPE), (dict(k=ap((3, 7, 2, 128), 3, gs.GS_I8), v=ap((3, 7, 2, 128), 3, gs.GS_I8)), gs.GS_ERR_DTYPE),
    (dict(k=ap((3, 7, 256), 2)), gs.GS_ERR_RANK), (dict(v=ap((3, 6, 2, 128), 3)), gs.GS_ERR_SHAPE), (dict(v=None), gs.GS_ERR_NULL),
])
def test_tokens_refuse(kw, status):
    L, a = gs.lib(), tokens(**kw)
    assert L.glenside_mx4_cache_append(*(ref(a[n]) for n in ("cache", "table", "first", "counts", "k", "v")), None) == status
    assert L.glenside_mx4_cache_read(*(ref(a[n]) for n in ("cache", "table", "first", "k", "v")), None) == status


@pytest.mark.parametrize("counts,status", [(ap((4,), 1, I32), gs.GS_ERR_SHAPE), (ap((3,), 1, gs.GS_F32), gs.GS_ERR_DTYPE), (ap((3,), 0, I32), gs.GS_ERR_RANK)])
def test_counts_refuse(counts, status):
    a = tokens(counts=counts)
    assert gs.lib().glenside_mx4_cache_append(*(ref(a[n]) for n in ("cache", "table", "first", "counts", "k", "v")), None) == status


def attention(**kw):
    a = dict(q=ap((3, 2, 8, 128), 3), cache=cache(), table=ap((3, 5), 1, I32), lengths=ap((3,), 1, I32), scale=1.0, window=0, sinks=0,
             out=ap((3, 2, 8, 128), 3), ws=None, bytes=0)
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(q=ap((3, 2, 8, 128), 3, gs.GS_F32)), gs.GS_ERR_DTYPE), (dict(q=ap((3, 2, 7, 128), 3)), gs.GS_ERR_SHAPE), (dict(q=ap((3, 2, 8, 64), 3)), gs.GS_ERR_SHAPE),
    (dict(q=ap((3, 16, 128), 2)), gs.GS_ERR_RANK), (dict(q=None), gs.GS_ERR_NULL), (dict(cache=cache(dim=100)), gs.GS_ERR_UNSUPPORTED),
    (dict(cache=cache(data=None)), gs.GS_ERR_NULL), (dict(table=ap((4, 5), 1, I32)), gs.GS_ERR_SHAPE), (dict(lengths=ap((2,), 1, I32)), gs.GS_ERR_SHAPE),
    (dict(lengths=ap((3,), 1, gs.GS_BF16)), gs.GS_ERR_DTYPE), (dict(lengths=None), gs.GS_ERR_NULL), (dict(scale=float("nan")), gs.GS_ERR_UNSUPPORTED),
    (dict(scale=float("inf")), gs.GS_ERR_UNSUPPORTED), (dict(window=-1), gs.GS_ERR_SHAPE), (dict(sinks=-1), gs.GS_ERR_SHAPE),
    (dict(out=ap((3, 2, 8, 128), 4)), gs.GS_ERR_RANK), (dict(out=ap((3, 1, 8, 128), 3)), gs.GS_ERR_SHAPE), (dict(out=ap((3, 2, 8, 128), 3, gs.GS_I32)), gs.GS_ERR_DTYPE),
    (dict(out=None), gs.GS_ERR_NULL),
    # a long table: parts of the sequence need a workspace
    (dict(table=ap((3, 500), 1, I32)), gs.GS_ERR_WORKSPACE), (dict(table=ap((3, 500), 1, I32), ws=FAKE, bytes=100), gs.GS_ERR_WORKSPACE),
    (dict(table=ap((3, 500), 1, I32), ws=FAKE + 4, bytes=1 << 30), gs.GS_ERR_WORKSPACE),
])
def test_attention_refuses(kw, status):
    a = attention(**kw)
    assert gs.lib().glenside_mx4_attend(ref(a["q"]), ref(a["cache"]), ref(a["table"]), ref(a["lengths"]), a["scale"], a["window"], a["sinks"],
                                        ref(a["out"]), a["ws"], a["bytes"], None) == status


def test_attention_workspace():
    L = gs.lib()
    need = L.glenside_mx4_attend_workspace(ref(ap((3, 2, 8, 128), 3)), ref(cache()), ref(ap((3, 500), 1, I32)))
    assert need > 0 and need % 4 == 0
    assert L.glenside_mx4_attend_workspace(ref(ap((3, 2, 8, 128), 3)), ref(cache()), ref(ap((3, 2), 1, I32))) == 0
    assert L.glenside_mx4_attend_workspace(ref(ap((3, 2, 7, 128), 3)), ref(cache()), ref(ap((3, 500), 1, I32))) == 0


def refused(status, call, *args, **kw):
    with pytest.raises(gs.GlensideError) as e:
        call(*args, **kw)
    assert e.value.status == status


def test_binding_refuses():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    m = gs.Mx4(torch.zeros(4, 2, 16, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8), (4, 64), 1)
    refused(gs.GS_ERR_DTYPE, gs.mx4_quantize, x.to(torch.int8))
    refused(gs.GS_ERR_RANK, gs.mx4_quantize, x, 3)
    refused(gs.GS_ERR_RANK, gs.mx4_quantize, x[0, 0])
    refused(gs.GS_ERR_SHAPE, gs.mx4_quantize, x, out=m._replace(shape=(4, 65), scales=torch.zeros(4, 8, dtype=torch.uint8), values=torch.zeros(4, 3, 16, dtype=torch.uint8)))
    refused(gs.GS_ERR_SHAPE, gs.mx4_dequantize, m._replace(shape=(4, 65)))          # more blocks than there are
    refused(gs.GS_ERR_SHAPE, gs.mx4_dequantize, m._replace(scales=torch.zeros(4, 2, dtype=torch.uint8)))
    refused(gs.GS_ERR_RANK, gs.mx4_dequantize, m._replace(n_access=3))
    refused(gs.GS_ERR_DTYPE, gs.mx4_dequantize, m, out_dtype=torch.int32)
    refused(gs.GS_ERR_SHAPE, gs.mx4_dot, m, m, out=torch.zeros(4, 5))
    refused(gs.GS_ERR_DTYPE, gs.mx4_weight_dot, x.float(), m)
    refused(gs.GS_ERR_RANK, gs.mx4_weight_dot, x, m, n_access=-1)
    with pytest.raises(ValueError):
        gs.mx4_quantize(x.t())
    with pytest.raises(ValueError):
        gs.mx4_dequantize(m._replace(values=torch.zeros(4, 2, 16)))
    with pytest.raises(ValueError):
        gs.mx4_dot(m, m._replace(values=torch.zeros(4, 2, 16, dtype=torch.uint8, device="meta")))
    for wrong in (x, (1, 2), None, "m"):
        with pytest.raises((TypeError, AttributeError)):
            gs.mx4_dequantize(wrong)
    with pytest.raises(TypeError):
        gs.mx4_dot(m, m, act=1.0)


def test_binding_refuses_caches():
    c = gs.mx4_cache(4, 2, 32, 64, "cpu")
    assert c.data.shape == (4, 2, 32 * 64 + 2 * 32 * 2) and not c.data.any()
    table, n = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    k = torch.zeros(3, 5, 2, 64, dtype=torch.bfloat16)
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_cache, 4, 2, 30, 64, "cpu")
    refused(gs.GS_ERR_SHAPE, gs.mx4_cache_append, c._replace(page_size=64), table, n, k, k)
    refused(gs.GS_ERR_SHAPE, gs.mx4_cache_append, c._replace(data=c.data[:, :, :-16].contiguous()), table, n, k, k)
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_cache_append, c._replace(page_size=17), table, n, k, k)
    refused(gs.GS_ERR_DTYPE, gs.mx4_cache_append, c, table.long().float(), n, k, k)
    refused(gs.GS_ERR_SHAPE, gs.mx4_cache_append, c, table, n[:2], k, k)
    refused(gs.GS_ERR_SHAPE, gs.mx4_cache_read, c, table, n, -1)
    refused(gs.GS_ERR_SHAPE, gs.mx4_cache_read, c, table, n, 4, k=k, v=k)
    refused(gs.GS_ERR_SHAPE, gs.mx4_attend, k[:, :, :, :32].contiguous(), c, table, n, 1.0)
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_attend, k, c, table, n, float("inf"))
    refused(gs.GS_ERR_SHAPE, gs.mx4_attend, k, c, table, n, 1.0, window=-2)
    with pytest.raises(ValueError):
        gs.mx4_attend(k.transpose(1, 2), c, table, n, 1.0)
    with pytest.raises(TypeError):
        gs.mx4_attend(k, c, table, n, "1")


@pytest.mark.parametrize("scale", [2.36e38, -2.36e38, 3.0e38, 3.4028234e38])
def test_attention_refuses_scales_whose_unit_is_infinite(scale):
    """Scores are computed times log2 e; up to that line a call gets as far as the check of its workspace."""
    for given, status in ((scale, gs.GS_ERR_UNSUPPORTED), (scale / abs(scale) * 2.358e38, gs.GS_ERR_WORKSPACE)):
        a = attention(table=ap((3, 500), 1, I32), scale=given)
        assert gs.lib().glenside_mx4_attend(ref(a["q"]), ref(a["cache"]), ref(a["table"]), ref(a["lengths"]), a["scale"], a["window"], a["sinks"],
                                            ref(a["out"]), a["ws"], a["bytes"], None) == status


def test_a_cache_without_pages():
    c = gs.mx4_cache(0, 2, 32, 64, "cpu")
    assert c.data.shape == (0, 2, 32 * 64 + 2 * 32 * 2) and (c.page_size, c.head_dim) == (32, 64)
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_cache, 0, 2, 30, 64, "cpu")
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_cache, -1, 2, 32, 64, "cpu")


@pytest.mark.parametrize("sizes", [(4, (1 << 32) + 2, 32, 64), (4, 2, (1 << 32) + 32, 64), (4, 2, 32, (1 << 32) + 64), ((1 << 64) + 4, 2, 32, 64),
                                   (4, 2 - (1 << 32), 32, 64)])
def test_a_cache_of_sizes_beyond_the_descriptor(sizes):
    """32 bits of such a size are a possible one."""
    refused(gs.GS_ERR_UNSUPPORTED, gs.mx4_cache, *sizes, "cpu")
