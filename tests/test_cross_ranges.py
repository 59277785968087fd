"""Into how many ranges of states a forward call of cross attention is cut, asked on the host (no GPU): what the ranges leave for the launch that
joins them is counted, and a launch stays within the limits that the entry points check."""
import ctypes
import random

import pytest

from test_cross_rules import BF16, F32, LIB, _Shape, plan


def scratch(dtype, *shape):
    f = LIB._ZN3moe19cross_scratch_bytesEiRKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_int, ctypes.c_void_p], ctypes.c_size_t
    return f(dtype, ctypes.byref(_Shape(*shape)))


# us of a call (projections of 8 columns) in that many ranges; 0: blocks of 128 columns
@pytest.mark.parametrize("dtype,shape,us", [
    (BF16, (10, 1162, 8161, 1, 1, 64), {0: 126.5, 1: 111.0, 2: 102.6, 4: 93.3, 8: 99.2, 16: 113.8, 32: 139.1, 64: 196.8}),
    (BF16, (19, 83, 8174, 8, 4, 64), {0: 127.0, 1: 113.8, 2: 117.3, 4: 117.4, 8: 121.7, 16: 136.2, 32: 168.8, 64: 250.8}),
    (BF16, (19, 15, 8100, 24, 3, 64), {0: 126.6, 1: 94.3, 2: 68.9, 4: 69.5, 8: 74.1, 16: 80.2, 32: 96.4, 64: 130.3}),
    (BF16, (6, 200, 4000, 2, 2, 128), {0: 94.9, 1: 69.2, 2: 43.6, 4: 45.9, 8: 42.3, 16: 53.3, 32: 71.6}),
    (BF16, (3, 1000, 4000, 2, 2, 64), {0: 67.0, 1: 48.2, 2: 40.0, 4: 38.1, 8: 40.0, 16: 48.6, 32: 62.1}),
    (BF16, (2, 300, 2000, 8, 8, 64), {0: 39.6, 1: 29.8, 2: 27.9, 4: 27.8, 8: 30.3, 16: 36.0}),
    (BF16, (1, 1, 8000, 16, 16, 128), {0: 163.9, 1: 128.7, 2: 73.9, 4: 44.6, 8: 32.1, 16: 29.5, 32: 34.1}),
    (F32, (19, 83, 8174, 8, 4, 64), {0: 761.9, 1: 381.0, 2: 382.9, 4: 382.4, 8: 371.7, 16: 380.0, 32: 431.6, 64: 570.9}),
    (F32, (1, 500, 8000, 2, 1, 128), {0: 1296.6, 1: 334.0, 2: 181.5, 4: 100.7, 8: 61.1, 16: 68.5, 32: 86.9})])
def test_ranges_of_a_call_as_measured(dtype, shape, us):
    few, splits = plan(dtype, *shape)
    assert us[splits if few else 0] <= 1.1 * min(us.values())


def accepted(r):
    """A shape that the entry points take (moe_cross_dims)."""
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))
    while True:
        kv_heads, share, d = log(1, 64), r.choice([1, 2, 4, 8, 16, 32]), r.choice([64, 128])
        B, Lq, Lk = log(1, 1 << 20), log(1, 1 << 24), log(1, 1 << 24)
        pairs = B * kv_heads
        if kv_heads * share * d >= 1 << 23 or B * Lk >= 1 << 30 or B * Lq >= 1 << 30 or Lq * share >= 1 << 29:
            continue
        if pairs * -(-Lq * share // 32) < 1 << 24 and pairs * -(-Lk // 32) < 1 << 24:
            return B, Lq, Lk, kv_heads * share, kv_heads, d


def test_launches_and_sums_of_ranges_are_bounded():
    """Less than 2^24 blocks of 256 threads of any call, and of a call in ranges no more than a few rounds of the device: 2048 blocks of 32 columns
    of 128 floats and two are 34 MB."""
    r = random.Random(3)
    for _ in range(20000):
        shape = accepted(r)
        B, Lq, Lk, heads, kv_heads, d = shape
        for dtype in (BF16, F32):
            few, splits = plan(dtype, *shape)
            if few:
                assert B * kv_heads * -(-Lq * (heads // kv_heads) // 32) * splits < 1 << 24, shape
            assert scratch(dtype, *shape) <= 2048 * 32 * (4 * 128 + 8) + 256, shape
