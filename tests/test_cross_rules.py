"""Which form a forward call of cross attention and a product of few rows take, asked on the host (no GPU): the one that was measured to be
the faster, at points on both sides of the lines; and which forms the GPU tests reach."""
import ctypes

import pytest

import paper_2006_16668_amd as moe
from test_gpu_cross_attention import CASES

LIB = ctypes.CDLL(moe.library_path())
BF16, F32 = 1, 0


class _Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_longlong)] + [(n, ctypes.c_int) for n in ("Lq", "Lk", "heads", "kv_heads", "d")]


class _Plan(ctypes.Structure):
    _fields_ = [("few", ctypes.c_bool), ("splits", ctypes.c_int)]


def plan(dtype, B, Lq, Lk, heads, kv_heads, d):
    f = LIB._ZN3moe10cross_planEiRKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_int, ctypes.c_void_p], _Plan
    s = _Shape(B, Lq, Lk, heads, kv_heads, d)
    p = f(dtype, ctypes.byref(s))
    return p.few, p.splits


# us of blocks of 128 columns, and of 32 in the best number of ranges
@pytest.mark.parametrize("dtype,shape,wide,few", [
    (BF16, (64, 1, 2048, 16, 16, 128), 120, 128), (BF16, (1, 4, 53, 16, 16, 128), 5.0, 6.1), (BF16, (1, 1, 1000, 16, 16, 128), 23.7, 10.1),
    (BF16, (1, 1, 8000, 16, 16, 128), 155, 23.0), (BF16, (8, 1, 1000, 16, 16, 128), 23.2, 19.1), (BF16, (4, 8, 4000, 16, 2, 128), 82, 13.7),
    (BF16, (4, 64, 1000, 8, 8, 128), 26.9, 14.2), (BF16, (3, 700, 700, 4, 4, 128), 20.4, 29.1), (BF16, (16, 1, 2000, 8, 8, 64), 28.2, 16.9),
    (BF16, (2, 300, 2000, 8, 8, 64), 34.5, 23.0), (BF16, (27, 834, 100, 8, 8, 64), 18.9, 47.2), (BF16, (32, 1024, 1024, 16, 16, 128), 340, 9999),
    (F32, (5, 187, 411, 8, 8, 64), 40.8, 16.3), (F32, (8, 500, 500, 8, 8, 64), 59.0, 63.8), (F32, (27, 834, 100, 8, 8, 64), 56.4, 95.4),
    (F32, (1, 1, 1000, 16, 16, 128), 165, 16.2), (F32, (16, 64, 256, 8, 8, 64), 28.5, 13.0), (F32, (32, 256, 256, 8, 8, 64), 55.0, 70.0)])
def test_form_of_a_call(dtype, shape, wide, few):
    assert plan(dtype, *shape)[0] == (few < wide)


def test_ranges_of_states():
    for dtype in (BF16, F32):
        for Lk in (1, 31, 128, 129, 1000, 8192, 1 << 20):
            for B in (1, 3, 64):
                few, splits = plan(dtype, B, 1, Lk, 4, 4, 128)
                assert 1 <= splits <= 64 and (few or splits == 1) and splits <= max(1, (Lk + 127) // 128)


def test_the_cases_reach_every_form():
    seen = {(dtype, *(lambda p: (p[0], p[1] > 1))(plan(dtype, *c[:6])), c[5]) for dtype in (BF16, F32) for c in CASES}
    assert seen == {(dtype, few, split, d) for dtype in (BF16, F32) for few, split in ((False, False), (True, False), (True, True)) for d in (64, 128)}


def ranges(B, Lq, Lk, heads, kv_heads, d):
    f = LIB._ZN3moe16cross_dkv_blocksERKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_void_p], ctypes.c_int
    s = _Shape(B, Lq, Lk, heads, kv_heads, d)
    all_, each = (Lq * (heads // kv_heads) + 63) // 64, f(ctypes.byref(s))
    assert 1 <= each <= all_
    return -(-all_ // each)


# us of dK and dV by one range of the columns, and by the best number of them with the launch that adds them up
@pytest.mark.parametrize("shape,one,more", [
    ((4, 2000, 1000, 8, 1, 128), 455, 87.4), ((4, 2000, 1000, 8, 1, 64), 295, 50.9), ((7, 1561, 66, 2, 1, 128), 93.0, 19.3),
    ((7, 1561, 66, 2, 1, 64), 61.1, 15.9), ((1, 2000, 60, 2, 2, 128), 62.6, 16.7), ((1, 1000, 500, 8, 8, 128), 36.1, 23.0),
    ((1, 1000, 500, 8, 8, 64), 23.8, 18.7), ((8, 1000, 100, 8, 8, 64), 24.4, 17.9), ((8, 1000, 100, 8, 8, 128), 36.7, 25.8),
    ((6, 900, 130, 4, 4, 64), 22.4, 15.6), ((1, 500, 500, 8, 8, 64), 14.5, 15.9), ((1, 500, 500, 8, 8, 128), 21.7, 22.4),
    ((2, 300, 2000, 8, 8, 64), 16.2, 23.6), ((2, 300, 2000, 8, 8, 128), 20.3, 46.0), ((4, 100, 100, 4, 4, 128), 10.0, 14.4),
    ((16, 200, 256, 8, 8, 128), 18.0, 42.7), ((27, 834, 100, 8, 8, 128), 35.2, 54.2), ((8, 1000, 1000, 8, 8, 64), 42.7, 64.5)])
def test_ranges_of_columns(shape, one, more):
    assert (ranges(*shape) > 1) == (more < one)


def test_ranges_run_at_once_and_none_is_empty():
    for d in (64, 128):
        for B in (1, 2, 7, 64, 300, 4000):
            for Lq in (1, 63, 64, 65, 1000, 4097, 1 << 20):
                for Lk in (1, 128, 129, 5000):
                    n = ranges(B, Lq, Lk, 4, 2, d)
                    all_ = (2 * Lq + 63) // 64
                    assert 1 <= n <= 32 and (n - 1) * -(-all_ // n) < all_
                    assert n == 1 or n * B * 2 * ((Lk + 127) // 128) <= (512 if d == 64 else 256)
    assert {(ranges(*c[:6]) > 1, c[5]) for c in CASES} == {(False, 64), (True, 64), (False, 128), (True, 128)}


# K, N, rows; us of the kernels for many rows and of this one
@pytest.mark.parametrize("dtype,K,N,rows,many,few", [
    (BF16, 1024, 2048, 1, 5.7, 3.4), (BF16, 1024, 2048, 128, 6.0, 4.4), (BF16, 1024, 2048, 192, 6.1, 7.2), (BF16, 2048, 1024, 256, 9.6, 6.1),
    (BF16, 1024, 4096, 64, 6.0, 4.6), (BF16, 1024, 4096, 96, 6.2, 7.3), (F32, 1024, 2048, 1, 16.6, 4.3), (F32, 1024, 2048, 96, 17.2, 12.5),
    (F32, 2048, 1024, 64, 29.3, 9.2), (F32, 2048, 4096, 64, 30.2, 31.1)])
def test_products_of_few_rows(dtype, K, N, rows, many, few):
    f = LIB._ZN3moe11few_rows_okEixi
    f.argtypes, f.restype = [ctypes.c_int, ctypes.c_longlong, ctypes.c_int], ctypes.c_bool
    assert f(dtype, rows, N) == (few < many)
    assert not f(dtype, 1 << 40, 64)
