"""Rules of the vocabulary's products, asked on the host (no GPU): each product takes the kernel that was measured to be the faster one,
and the cases of the GPU tests reach every kernel."""
import ctypes

import pytest

import paper_2006_16668_amd as moe
from test_gpu_vocab_loss import CE, KD

LIB = ctypes.CDLL(moe.library_path())


class DxPlan(ctypes.Structure):
    _fields_ = [("splits", ctypes.c_int), ("k", ctypes.c_int), ("tiles", ctypes.c_bool)]


def _f(mangled, restype, n):
    f = getattr(LIB, mangled)
    f.restype, f.argtypes = restype, [ctypes.c_int] * n
    return f


_on_tiles = _f("_ZN3moe21vocab_logits_on_tilesEiiibd", ctypes.c_bool, 4)
_on_tiles.argtypes = [ctypes.c_int] * 4 + [ctypes.c_double]


def logits_on_tiles(rows, entries, M, pack, saved=0.0):
    return _on_tiles(rows, entries, M, pack, saved)


dx_plan = _f("_ZN3moe13vocab_dx_planEiii", DxPlan, 3)
dw_splits_f32 = _f("_ZN3moe19vocab_dw_splits_f32Eiii", ctypes.c_int, 3)
_dw_splits = LIB["_ZN3moe15vocab_dw_splitsEiiiRKNS_11VocabDxPlanE"]
_dw_splits.argtypes = [ctypes.c_int] * 3 + [ctypes.POINTER(DxPlan)]


def dw_splits(rows, entries, M):
    return _dw_splits(rows, entries, M, ctypes.byref(dx_plan(rows, entries, M)))


dw_on_tiles = _f("_ZN3moe17vocab_dw_on_tilesEiii", ctypes.c_bool, 3)


# M, rows, entries, us of z and of dw in the edge kernel and on 256 x 256 tiles
@pytest.mark.parametrize("M,rows,entries,z_edge,z_tiles,dw_edge,dw_tiles", [
    (256, 1024, 20000, 25.5, 28.5, 19.1, 26.3), (256, 6000, 100000, 284.8, 263.2, 245.5, 156.1), (512, 256, 5000, 8.3, 19.2, 5.9, 11.8),
    (512, 2048, 32000, 97.0, 79.8, 73.5, 59.6), (512, 6000, 5000, 50.5, 42.6, 63.4, 106.4), (1024, 1024, 32000, 83.4, 64.2, 76.6, 63.1),
    (1024, 2048, 20000, 102.8, 89.6, 86.5, 96.5), (1024, 6000, 32000, 476.0, 368.9, 434.4, 324.2), (2048, 256, 1000, 11.9, 40.7, 5.2, 11.6),
    (2048, 512, 32000, 83.4, 59.6, 80.2, 73.2), (2048, 1024, 100000, 534.9, 369.9, 483.1, 398.1)])
def test_faster_kernel(M, rows, entries, z_edge, z_tiles, dw_edge, dw_tiles):
    assert logits_on_tiles(rows, entries, M, False) == (z_tiles < z_edge)
    assert dw_on_tiles(rows, entries, M) == (dw_tiles < dw_edge)


def test_plans_cover_the_vocabulary():
    for rows in (1, 7, 64, 300, 2048, 32768):
        for entries in (1, 63, 64, 300, 5000, 50257, 200000):
            for M in (8, 776, 1024, 4096):
                p = dx_plan(rows, entries, M)
                assert 1 <= p.splits <= 64 and p.k % 64 == 0 and (p.splits - 1) * p.k < entries <= p.splits * p.k


def test_cases_reach_every_kernel():
    seen = set()
    for G, S, M, V, dtype, empty, piece in CE:
        if dtype != "bf16":
            continue
        n, N = min(V, piece or V), G * S
        seen |= {("z", logits_on_tiles(N, V, M, True)), ("dz", logits_on_tiles(N, n, M, False)), ("dx", dx_plan(N, n, M).tiles),
                 ("dx ranges", dx_plan(N, n, M).splits > 1), ("dw", dw_on_tiles(N, n, M))}
        # sums whose length is no multiple of a step, and few rows with a target, on tiles
        if logits_on_tiles(N, n, M, False):
            seen |= {("dz tail", M % 64 != 0), ("dz empty", empty > 0.5)}
        if dx_plan(N, n, M).tiles:
            seen.add(("dx tail", n % 64 != 0 or V % n % 64 != 0))
    assert seen == {(k, b) for k in ("z", "dz", "dx", "dx ranges", "dw", "dz tail", "dz empty") for b in (True, False)} | \
        {("dx tail", b) for b in (True, False)}
    # the product leaves the logits at a teacher's entries: more than 100 MB of w's rows, on tiles in any case or because of them
    sorts = [(G * S, V, M, True, 2 * G * S * K * M / 6e6 - 16) for G, S, M, V, K, T, dtype, e, p in KD
             if dtype == "bf16" and 2 * G * S * K * M > 1e8]
    assert {logits_on_tiles(*s[:4]) for s in sorts if logits_on_tiles(*s)} == {True, False}


def test_ranges_of_the_rows():
    """A small vocabulary's dw is summed over ranges of many tokens, and such are among the cases: all rows, hardly any, pieces."""
    for f in (dw_splits, dw_splits_f32):
        assert all(f(N, 300, 64) == 1 for N in (1, 64, 300)) and f(32768, 300, 128) > 8
        assert all(1 <= f(N, V, M) <= 32 for N in (1, 700, 5000, 32768) for V in (1, 200, 3000, 50257) for M in (8, 256, 2048))
    # (two launches where one for both gradients is faster)
    assert dw_splits(1878, 242, 1008) == 1 and dw_splits(4222, 3434, 312) == 1 and dw_splits(11656, 863, 472) > 1
    for dtype, f in (("bf16", dw_splits), ("f32", dw_splits_f32)):
        ranged = [(empty > 0.9, piece > 0) for G, S, M, V, dt, empty, piece in CE if dt == dtype and f(G * S, min(V, piece or V), M) > 1]
        assert {(False, False), (True, False), (False, True)} <= set(ranged)
        assert f(9000, 300, 64) > 1


def test_what_the_entry_points_refuse():
    sh = moe.MoEShape(1, 8, 64, 64, 2, 1, "bf16")
    for dims, status in ((moe.VocabDims(0), -1), (moe.VocabDims(-5), -1), (moe.VocabDims(100, piece=-1), -1), (moe.VocabDims((1 << 23) + 1), -2)):
        for f in (moe.moe_vocab_workspace_bytes, moe.moe_vocab_backward_workspace_bytes):
            with pytest.raises(moe.MoEError) as e:
                f(sh, dims)
            assert e.value.status == status
    for bad, status in ((moe.MoEShape(1, 8, 63, 64, 2, 1, "bf16"), -2), (moe.MoEShape(1, 8, 66, 64, 2, 1, "f32"), -2),
                        (moe.MoEShape(16, 1 << 20, 64, 64, 2, 1, "bf16"), -2), (moe.MoEShape(0, 8, 64, 64, 2, 1, "bf16"), -1)):
        with pytest.raises(moe.MoEError) as e:
            moe.moe_vocab_workspace_bytes(bad, moe.VocabDims(100))
        assert e.value.status == status
    with pytest.raises(moe.MoEError) as e:
        moe.moe_layer_norm_backward_workspace_bytes(moe.MoEShape(1, 0, 64, 64, 2, 1, "bf16"))
    assert e.value.status == -1


class _C(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("G", "S", "M", "H", "E", "C", "act_dtype")]


class _D(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("K", ctypes.c_int32), ("piece", ctypes.c_int32), ("temperature", ctypes.c_float)]


def test_argument_checks_of_the_c_calls():
    """Pointers are checked before anything is enqueued; the addresses below are never followed."""
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    cfg, ok, ws = _C(1, 8, 64, 64, 2, 1, 1), 4096, 1 << 16

    def distill(dims, *over, ws_bytes=1 << 30, n=8):
        args = [ok] * n
        for i, v in over:
            args[i] = v
        f = LIB.moe_vocab_distill
        f.argtypes, f.restype = [vp, vp] + [vp] * 8 + [sz, vp], ctypes.c_int
        return f(ctypes.byref(cfg), ctypes.byref(dims), *[vp(a) for a in args], sz(ws_bytes), None)

    good = _D(100, 4, 0, 1.0)
    for i in range(8):
        assert distill(good, (i, 0)) == -1, i                   # null
        assert distill(good, (i, 4104)) == -1, i                # not 16-byte aligned
    assert distill(good, (7, 4112)) == -1                       # a workspace at less than 256 bytes
    assert distill(good, ws_bytes=100) == -3
    for dims, status in ((_D(100, 0, 0, 1.0), -1), (_D(100, 257, 0, 1.0), -2), (_D(100, 4, 0, 0.0), -1), (_D(100, 4, 0, -1.0), -1),
                         (_D(100, 4, 0, float("nan")), -1), (_D(100, 4, 0, float("inf")), -1), (_D(100, 4, 0, 1e-45), -1)):
        assert distill(dims, ws_bytes=100) == status

    def call(name, n, missing, dims=good):
        f = getattr(LIB, name)
        f.argtypes, f.restype = [vp, vp] + [vp] * n + [sz, vp], ctypes.c_int
        args = [ok] * n
        if missing is not None:
            args[missing] = 0
        return f(ctypes.byref(cfg), ctypes.byref(dims), *[vp(a) for a in args], sz(100), None)

    for name, n in (("moe_vocab_loss", 6), ("moe_vocab_loss_backward", 9), ("moe_vocab_distill_backward", 10)):
        assert all(call(name, n, i) == -1 for i in range(n)), name
        assert call(name, n, None) == -3, name
    f = LIB.moe_add_layer_norm_backward
    f.argtypes, f.restype = [vp] * 9 + [sz, vp], ctypes.c_int
    for i in (0, 1, 2, 4, 5, 6, 7):
        args = [ok] * 8
        args[i] = 0
        assert f(ctypes.byref(cfg), *[vp(a) for a in args], sz(1 << 30), None) == -1
    assert f(ctypes.byref(cfg), *[vp(ok)] * 8, sz(10), None) == -3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspace_without_teacher_ignores_its_entries(dtype):
    """K is not read for a cross entropy: whatever stands there, the sizes asked for serve one.  The size of a distillation's, large
    enough for its entries to be sorted, grows with K."""
    sh = moe.MoEShape(1, 8192, 1024, 64, 2, 1, dtype)
    for f in (moe.moe_vocab_workspace_bytes, moe.moe_vocab_backward_workspace_bytes):
        plain = f(sh, moe.VocabDims(64000))
        assert all(f(sh, moe.VocabDims(64000, K=K)) == plain for K in (-1, -(1 << 31), 257, (1 << 31) - 1))
        assert plain <= f(sh, moe.VocabDims(64000, K=32)) <= f(sh, moe.VocabDims(64000, K=256)) < plain + (1 << 26)


def test_tensors_of_another_kind_are_refused():
    import torch
    sh, d = moe.MoEShape(1, 8, 64, 64, 2, 1, "bf16"), moe.VocabDims(100)
    host = torch.zeros(1)
    with pytest.raises(TypeError):
        moe.moe_vocab_loss(sh, d, None, host, host, host, host, host)
