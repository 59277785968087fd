"""Which calls of cross attention carry q and ctx as pairs of bf16, asked on the host (no GPU), and that the GPU tests reach every form of them."""
import ctypes

import pytest

import paper_2006_16668_amd as moe
from test_cross_ranges import scratch
from test_cross_rules import BF16, LIB, _Plan, _Shape
from test_gpu_cross_few_tokens import CASES, GRADIENT_CASES


def pair_plan(*shape):
    f = LIB._ZN3moe15cross_pair_planERKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_void_p], _Plan
    p = f(ctypes.byref(_Shape(*shape)))
    return p.few, p.splits


def pair_ok(rows, N):
    f = LIB._ZN3moe16few_rows_pair_okExi
    f.argtypes, f.restype = [ctypes.c_longlong, ctypes.c_int], ctypes.c_bool
    return f(rows, N)


def in_pairs(B, Lq, Lk, M, heads, kv_heads, d):
    """From the workspace of an inference: one array of q and one of ctx more, and the scratch of the other plan."""
    sh, dims, shape = moe.MoEShape(B, Lq, M, 64, 2, 1), moe.CrossDims(B, Lq, Lk, heads, d, kv_heads), (B, Lq, Lk, heads, kv_heads, d)
    f = LIB._ZN3moe24cross_pair_scratch_bytesERKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_void_p], ctypes.c_size_t
    up = lambda n: (n + 255) // 256 * 256
    array, got = up(2 * B * Lq * heads * d), moe.moe_cross_workspace_bytes(sh, dims)
    assert got in (2 * array + up(scratch(BF16, *shape)), 4 * array + up(f(ctypes.byref(_Shape(*shape)))))
    return got == 4 * array + up(f(ctypes.byref(_Shape(*shape))))


def test_the_cases_reach_every_form():
    for B, Lq, Lk, M, heads, kv_heads, d, _ in CASES:
        rows = B * Lq
        assert pair_ok(rows, M) and -(-rows // 32) * -(-heads * d // 32) <= 256 and in_pairs(B, Lq, Lk, M, heads, kv_heads, d)
    seen = {(*(lambda p: (p[0], p[1] > 1))(pair_plan(*c[:3], *c[4:7])), c[6]) for c in CASES}
    assert seen == {(few, split, d) for few, split in ((False, False), (True, False), (True, True)) for d in (64, 128)}


def pair_ranges(B, Lq, Lk, heads, kv_heads, d):
    f = LIB._ZN3moe21cross_pair_dkv_blocksERKNS_10CrossShapeE
    f.argtypes, f.restype = [ctypes.c_void_p], ctypes.c_int
    all_, each = (Lq * (heads // kv_heads) + 63) // 64, f(ctypes.byref(_Shape(B, Lq, Lk, heads, kv_heads, d)))
    assert 1 <= each <= all_
    return -(-all_ // each)


def test_the_gradients_cases_reach_every_form():
    """Ranges of columns or none, sources of up to 64 states and more."""
    for B, Lq, Lk, M, heads, kv_heads, d, _ in GRADIENT_CASES:
        assert in_pairs(B, Lq, Lk, M, heads, kv_heads, d)
    seen = {(pair_ranges(*c[:3], *c[4:7]) > 1, c[2] > 64, c[6]) for c in GRADIENT_CASES}
    assert {(r, d) for r, _, d in seen} == {(r, d) for r in (False, True) for d in (64, 128)} and {(f, d) for _, f, d in seen} == {(f, d) for f in (False, True) for d in (64, 128)}


# us of the kernels in that many ranges of blocks of 16 columns; 0: blocks of 64
@pytest.mark.parametrize("shape,us", [
    ((55, 4, 131, 8, 8, 128), {0: 9.3, 1: 14.3, 2: 25.0}), ((47, 1, 267, 16, 16, 128), {0: 26.0, 1: 34.4, 2: 46.5}), ((1, 2, 23, 3, 3, 128), {0: 5.1, 1: 7.0}),
    ((4, 1, 55, 3, 3, 64), {0: 4.1, 1: 4.9}), ((11, 1, 43, 2, 2, 128), {0: 5.4, 1: 7.0}), ((57, 1, 240, 4, 4, 64), {0: 7.3, 1: 6.2, 2: 10.8}),
    ((106, 1, 633, 2, 2, 64), {0: 12.8, 1: 9.6, 2: 13.7, 4: 16.3}), ((1, 16, 115, 4, 4, 128), {0: 7.3, 1: 6.2}), ((4, 1, 87, 16, 2, 128), {0: 6.9, 1: 5.8}),
    ((5, 16, 2183, 16, 16, 128), {0: 52.5, 1: 34.9, 2: 27.9, 4: 33.1, 8: 35.4, 16: 42.4}), ((83, 4, 2954, 2, 2, 64), {0: 46.9, 1: 31.5, 2: 27.9, 4: 31.6, 8: 32.3, 16: 35.9}),
    ((14, 1, 2193, 32, 4, 128), {0: 51.3, 1: 34.2, 2: 25.6, 4: 21.5, 8: 25.9, 16: 33.2}), ((30, 7, 2018, 3, 3, 64), {0: 32.9, 1: 20.8, 2: 19.6, 4: 16.3, 8: 18.3, 16: 19.9}),
    ((8, 12, 2761, 4, 4, 128), {0: 63.1, 1: 39.5, 2: 27.9, 4: 20.9, 8: 17.7, 16: 22.0}), ((9, 1, 3756, 8, 2, 128), {0: 80.3, 1: 50.0, 2: 33.1, 4: 22.3, 8: 16.2, 16: 19.7}),
    ((3, 4, 5147, 3, 3, 128), {0: 108.5, 1: 65.8, 2: 41.4, 4: 26.0, 8: 18.7, 16: 14.6, 32: 17.0}), ((7, 1, 5269, 8, 4, 64), {0: 77.2, 1: 48.0, 2: 31.6, 4: 21.0, 8: 17.0, 16: 15.0, 32: 18.4})])
def test_form_of_a_call_in_pairs(shape, us):
    few, splits = pair_plan(*shape)
    assert us[splits if few else 0] <= 1.15 * min(us.values())


@pytest.mark.parametrize("rows,N,ok", [(1, 8, True), (16, 8192, True), (17, 8192, False), (128, 1024, True), (129, 1024, False), (4096, 32, True), (4097, 32, False),
                                       (1 << 40, 8, False)])
def test_products_of_pairs_fill_the_device_once(rows, N, ok):
    assert pair_ok(rows, N) == ok


def test_steps_of_generation_are_in_pairs_and_batches_of_training_are_not():
    for B in (1, 4, 64, 128):
        assert in_pairs(B, 1, 2048, 1024, 16, 16, 128)
    assert in_pairs(1, 128, 300, 64, 1, 1, 64) and not in_pairs(1, 129, 300, 64, 1, 1, 64)
    assert not in_pairs(129, 1, 300, 1024, 16, 16, 128) and not in_pairs(32, 1024, 1024, 1024, 16, 16, 128)
    # (fp32 has no pairs)
    sh, dims = moe.MoEShape(4, 1, 1024, 64, 2, 1, "f32"), moe.CrossDims(4, 1, 53, 16, 128)
    assert moe.moe_cross_workspace_bytes(sh, dims) == 2 * 4 * 2048 * 4 + (scratch(0, 4, 1, 53, 16, 16, 128) + 255) // 256 * 256
