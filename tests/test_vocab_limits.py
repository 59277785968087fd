"""Sizes and temperatures at the ends of what the vocabulary's losses take, asked on the host (no GPU)."""
import pytest

import paper_2006_16668_amd as moe


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
