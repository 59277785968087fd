"""Sizes and temperatures at the ends of what the vocabulary's losses take, asked on the host (no GPU)."""
import ctypes

import pytest

import paper_2006_16668_amd as moe
from test_vocab_rules import LIB, _C, _D


def test_rows_packed_by_fewer_threads_than_a_launch_has():
    """The backward pass packs whole 64 rows, a thread per 16 bytes, and a launch has less than 2^32 threads: 16383 rows of 4 MB are
    below that, the 16384 that are packed are not."""
    f32 = lambda n: moe.MoEShape(1, n, 1 << 20, 64, 2, 1, "f32")
    dims = moe.VocabDims(256)
    for n in (16321, 16383):
        with pytest.raises(moe.MoEError) as e:
            moe.moe_vocab_backward_workspace_bytes(f32(n), dims)
        assert e.value.status == -2
    assert moe.moe_vocab_backward_workspace_bytes(f32(16320), dims) > 1 << 36
    # (neither the forward pass nor bf16 rows, of half the size, are packed by that many)
    assert moe.moe_vocab_workspace_bytes(f32(16383), dims) < 1 << 20
    assert moe.moe_vocab_backward_workspace_bytes(moe.MoEShape(1, 16383, 1 << 20, 64, 2, 1, "bf16"), dims) > 1 << 36


@pytest.mark.parametrize("temperature,status", [(3e-39, -1), (4.2e-39, -1), (4.3e-39, -3), (1.0, -3), (3e38, -3)])
def test_temperatures_whose_scale_is_a_number(temperature, status):
    """The logits' scale is log2(e) / T: with T below 4.24e-39 (log2(e) / 3.4e38) it is no finite number, which would make NaN of a logit of 0.
    (-3: the workspace is too small, all else is accepted; no address is followed.)"""
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    cfg, dims = _C(1, 8, 64, 64, 2, 1, 1), _D(100, 4, 0, temperature)
    for name, n in (("moe_vocab_distill", 8), ("moe_vocab_distill_backward", 10)):
        f = getattr(LIB, name)
        f.argtypes, f.restype = [vp, vp] + [vp] * n + [sz, vp], ctypes.c_int
        assert f(ctypes.byref(cfg), ctypes.byref(dims), *[vp(4096)] * n, sz(100), None) == status
