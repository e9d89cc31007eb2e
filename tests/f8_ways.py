"""Sizes at which products of scaled 8-bit floats are done in each of their ways: way, workgroups that share a sum, rows, columns, K,
experts (0: one matrix).  The ways are numbered as the library does (rows of w through registers, one and two tiles to a workgroup;
tiles of 32x64, 64x64, 64x128, 128x128 with eight waves and with four, 128x256, 256x256)."""

import ctypes

from paper_2105_09377_amd import binding as gs

WAYS = [
    (0, 1, 3, 40, 300, 0), (0, 1, 16, 500, 2100, 0), (1, 1, 9, 8200, 300, 0),
    (2, 1, 40, 100, 900, 0), (2, 1, 17, 33, 130, 0), (2, 2, 20, 70, 2922, 0), (2, 4, 19, 65, 4449, 0),
    (3, 1, 4118, 208, 130, 0), (3, 2, 4424, 51, 4952, 0), (3, 4, 2171, 50, 4159, 0),
    (4, 1, 356, 2933, 924, 0), (4, 4, 2120, 67, 4009, 0),
    (5, 1, 2557, 1222, 266, 0), (5, 4, 4257, 86, 5318, 0),
    (6, 1, 2883, 2436, 140, 0), (7, 1, 1175, 3522, 794, 0), (8, 1, 4447, 3039, 434, 0),
    (0, 1, 20, 100, 600, 8), (1, 1, 40, 2817, 300, 8), (2, 1, 36, 70, 300, 4), (3, 1, 4485, 195, 130, 8), (4, 1, 2093, 863, 146, 8),
    (5, 1, 2252, 1335, 263, 8), (6, 1, 3297, 2075, 130, 8), (7, 1, 4232, 723, 828, 40), (8, 1, 3416, 3641, 486, 4),
]


def plan(m, n, k, experts):
    f = gs.lib().gs_test_f8_dot_plan
    f.argtypes = [ctypes.c_int64] * 4 + [ctypes.POINTER(ctypes.c_int)]
    p = (ctypes.c_int * 2)()
    assert f(m, n, k, experts, p) == gs.GS_OK
    return tuple(p)
