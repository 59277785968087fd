"""What the decoder's and the losses' entry points refuse, asked on the host (no GPU): no address below is followed."""
import ctypes

import pytest

import paper_2006_16668_amd as moe
from paper_2006_16668_amd.binding import _CrossDims, _Gradient, _PolicyDims, _PreferenceDims
from test_vocab_rules import LIB, _C

VP, SZ = ctypes.c_void_p, ctypes.c_size_t
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
CFG = _C(2, 8, 64, 64, 2, 1, 1)


def cross(B=2, Lq=8, Lk=5, heads=4, kv_heads=2, d=64):
    return _CrossDims(B, Lq, Lk, heads, kv_heads, d)


def call(name, cfg, dims, args):
    """args: addresses, sizes in place of workspace lengths."""
    f = getattr(LIB, name)
    f.restype = ctypes.c_int
    f.argtypes = [VP, VP] + [SZ if isinstance(a, SZ) else VP for a in args]
    return f(ctypes.byref(cfg) if cfg is not None else None, ctypes.byref(dims) if dims is not None else None, *args)


def forward(cfg=CFG, dims=None, at=None, bytes_=0, name="moe_cross_attention"):
    args = [VP(4096)] * 7 + [SZ(bytes_), None]
    for i, v in (at or {}).items():
        args[i] = VP(v)
    return call(name, cfg, dims or cross(), args)


def backward(cfg=CFG, dims=None, at=None, fwd=0, ws=0):
    args = [VP(4096)] * 9 + [SZ(fwd)] + [VP(4096)] * 6 + [SZ(ws), None]
    for i, v in (at or {}).items():
        args[i] = VP(v)
    return call("moe_cross_attention_backward", cfg, dims or cross(), args)


@pytest.mark.parametrize("dims,status", [
    (cross(B=3), EINVAL), (cross(Lq=0, B=0), EINVAL), (cross(Lk=0), EINVAL), (cross(heads=4, kv_heads=3), EINVAL), (cross(kv_heads=0), EINVAL),
    (cross(heads=-4), EINVAL), (cross(d=32), EUNSUPPORTED), (cross(d=96), EUNSUPPORTED), (cross(heads=6, kv_heads=2), EUNSUPPORTED),
    (cross(heads=64, kv_heads=1), EUNSUPPORTED), (cross(heads=1 << 17, kv_heads=1 << 17), EUNSUPPORTED), (cross(Lk=1 << 30), EUNSUPPORTED),
    (cross(Lk=1 << 28), EUNSUPPORTED), (cross(Lk=(1 << 27) + 1, heads=64, kv_heads=64), EUNSUPPORTED)])
def test_shapes_of_cross_attention(dims, status):
    n = SZ()
    for name in ("moe_cross_workspace_bytes", "moe_cross_train_workspace_bytes", "moe_cross_backward_workspace_bytes"):
        assert call(name, CFG, dims, [ctypes.cast(ctypes.pointer(n), VP)]) == status
    assert forward(dims=dims) == forward(dims=dims, name="moe_cross_attention_train") == backward(dims=dims) == status
    assert call("moe_cross_keys", CFG, dims, [VP(4096)] * 3 + [None]) == status


def test_sizes_at_the_ends_of_what_a_launch_takes():
    """Blocks of 256 threads: less than 2^24 of them, by columns and by states."""
    n = SZ()
    at = [ctypes.cast(ctypes.pointer(n), VP)]
    for (G, S, dims, status) in (((1 << 20) - 1, 1, cross(B=(1 << 20) - 1, Lq=1, Lk=1, heads=16, kv_heads=16), 0),
                                 (1 << 20, 1, cross(B=1 << 20, Lq=1, Lk=1, heads=16, kv_heads=16), EUNSUPPORTED),
                                 (1, (1 << 25) - 32, cross(B=1, Lq=(1 << 25) - 32, Lk=1, heads=16, kv_heads=16), 0),
                                 (1, (1 << 25) - 31, cross(B=1, Lq=(1 << 25) - 31, Lk=1, heads=16, kv_heads=16), EUNSUPPORTED),
                                 (1, 1, cross(B=1, Lq=1, Lk=(1 << 25) - 32, heads=16, kv_heads=16), 0),
                                 (1, 1, cross(B=1, Lq=1, Lk=(1 << 25) - 31, heads=16, kv_heads=16), EUNSUPPORTED),
                                 (1, 1 << 24, cross(B=1, Lq=1 << 24, Lk=1, heads=32, kv_heads=1), EUNSUPPORTED)):
        for name in ("moe_cross_workspace_bytes", "moe_cross_train_workspace_bytes", "moe_cross_backward_workspace_bytes"):
            assert call(name, _C(G, S, 64, 64, 2, 1, 1), dims, at) == status, (name, G, S)


def test_arguments_of_cross_attention():
    assert forward() == backward() == EWORKSPACE
    for i in (0, 1, 3, 4, 5, 6):
        assert forward(at={i: 0}) == forward(at={i: 4097 if i != 6 else 4096 + 16}) == EINVAL
    assert forward(at={2: 0}) == EWORKSPACE and forward(at={2: 4098}) == EINVAL          # (no lengths; lengths off their 4 bytes)
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 10, 11, 12, 13, 14, 15):
        assert backward(at={i: 0}) == EINVAL, i
    assert backward(at={8: 4096 + 16}) == backward(at={15: 4096 + 128}) == EINVAL
    sh, dims = moe.MoEShape(2, 8, 64, 64, 2, 1), moe.CrossDims(2, 8, 5, 4, 64, 2)
    f, w = moe.moe_cross_train_workspace_bytes(sh, dims), moe.moe_cross_backward_workspace_bytes(sh, dims)
    assert backward(fwd=f - 1, ws=w) == backward(fwd=f, ws=w - 1) == EWORKSPACE
    for i in range(3):
        args = [VP(4096)] * 3 + [None]
        args[i] = VP(0)
        assert call("moe_cross_keys", CFG, cross(), args) == EINVAL
    assert forward(cfg=None) == forward(cfg=_C(2, 8, 60, 64, 2, 1, 1)) + 1 == EINVAL
    bad = ctypes.c_void_p()
    assert call("moe_cross_workspace_bytes", CFG, cross(), [bad]) == EINVAL


def test_workspaces_grow_with_the_calls():
    sh = moe.MoEShape(32, 1024, 1024, 64, 2, 1)
    dims = moe.CrossDims(32, 1024, 1024, 16, 128)
    n, rows = 32 * 1024 * 2048 * 2, 32 * 1024
    assert 2 * n <= moe.moe_cross_workspace_bytes(sh, dims)
    assert 2 * n + rows * 16 * 4 <= moe.moe_cross_train_workspace_bytes(sh, dims)
    assert 2 * n + 2 * n + rows * 1024 * 2 <= moe.moe_cross_backward_workspace_bytes(sh, dims)


def test_more_pairs_than_a_launch_takes():
    for P, status in (((1 << 24) - 1, EINVAL), (1 << 24, EUNSUPPORTED)):       # (a missing address, found after)
        assert call("moe_preference_loss", CFG, _PreferenceDims(P, 9, 0, 0.1, 0.0), [VP(0)] * 6 + [None]) == status


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("d", [(0, 9, 0, 0.1, 0.0), (-1, 9, 0, 0.1, 0.0), (1, 0, 0, 0.1, 0.0), (1, 9, 2, 0.1, 0.0), (1, 9, -1, 0.1, 0.0), (1, 9, 0, 0.0, 0.0),
                               (1, 9, 0, -1.0, 0.0), (1, 9, 0, NAN, 0.0), (1, 9, 1, INF, 0.0), (1, 9, 0, 0.1, 1.0), (1, 9, 0, 0.1, -0.1), (1, 9, 0, 0.1, NAN)])
def test_preferences_refused(d):
    assert call("moe_preference_loss", CFG, _PreferenceDims(*d), [VP(4096)] * 6 + [None]) == EINVAL
    assert call("moe_preference_loss_backward", CFG, _PreferenceDims(*d), [VP(4096)] * 5 + [None]) == EINVAL


@pytest.mark.parametrize("d", [(0, 0, 0.2, 0.2, 0.0), (9, 2, 0.2, 0.2, 0.0), (9, 0, -0.1, 0.2, 0.0), (9, 0, 1.1, 0.2, 0.0), (9, 0, NAN, 0.2, 0.0), (9, 0, 0.2, -0.1, 0.0),
                               (9, 0, 0.2, INF, 0.0), (9, 0, 0.2, NAN, 0.0), (9, 0, 0.2, 0.2, -1.0), (9, 0, 0.2, 0.2, NAN), (9, 0, 0.2, 0.2, INF)])
def test_policies_refused(d):
    for name in ("moe_policy_loss", "moe_policy_loss_backward"):
        assert call(name, CFG, _PolicyDims(*d), [VP(4096)] * 7 + [None]) == EINVAL


@pytest.mark.parametrize("beta", [3.5e38, 1e39, 1e300])
def test_weights_of_the_kl_term_past_fp32(beta):
    """The term is formed in fp32: such a weight would be infinite there, and the loss of a token whose term is 0 NaN."""
    for name in ("moe_policy_loss", "moe_policy_loss_backward"):
        assert call(name, CFG, _PolicyDims(9, 0, 0.2, 0.2, beta), [VP(4096)] * 7 + [None]) == EINVAL


def test_addresses_of_the_losses():
    pd, qd = _PreferenceDims(2, 9, 0, 0.1, 0.0), _PolicyDims(9, 1, 0.2, 0.2, 0.1)
    for name, dims, n, optional in (("moe_preference_loss", pd, 6, ()), ("moe_preference_loss_backward", pd, 5, ()), ("moe_policy_loss", qd, 7, (6,)),
                                    ("moe_policy_loss_backward", qd, 7, ())):
        for i in range(n):
            for bad in (0, 4097, 4104):
                if i in optional and bad == 0:
                    continue
                args = [VP(4096)] * n + [None]
                args[i] = VP(bad)
                assert call(name, CFG, dims, args) == EINVAL, (name, i, bad)
        assert call(name, None, dims, [VP(4096)] * n + [None]) == call(name, CFG, None, [VP(4096)] * n + [None]) == EINVAL


def _norm(list_, n, norm=4096, ws=4096, bytes_=0):
    f = LIB.moe_gradient_norm
    f.argtypes, f.restype = [VP, ctypes.c_int32, VP, VP, SZ, VP], ctypes.c_int
    return f(list_, n, VP(norm), VP(ws), SZ(bytes_), None)


def _clip(list_, n, norm=4096, limit=1.0):
    f = LIB.moe_clip_gradients
    f.argtypes, f.restype = [VP, ctypes.c_int32, VP, ctypes.c_double, VP], ctypes.c_int
    return f(list_, n, VP(norm), limit, None)


@pytest.mark.parametrize("entry,read,written", [((4096, 4096, -1, 0), EINVAL, EINVAL), ((4096, 4096, 8, 2), EINVAL, EINVAL), ((0, 4096, 8, 0), EINVAL, EINVAL),
                                                ((4098, 4096, 8, 1), EINVAL, EINVAL), ((4096, 0, 8, 1), EWORKSPACE, EINVAL), ((4096, 4104, 8, 1), EWORKSPACE, EINVAL),
                                                ((4096, 4096, (1 << 42) + 1, 1), EUNSUPPORTED, EUNSUPPORTED)])
def test_gradients_refused(entry, read, written):
    one = (_Gradient * 1)(_Gradient(*entry))
    assert _norm(one, 1) == read and _clip(one, 1) == written


def test_arguments_of_norm_and_clip():
    one = (_Gradient * 1)(_Gradient(4096, 4096, 8, 0))
    assert _norm(None, 1) == _norm(one, -1) == _clip(None, 1) == _clip(one, -1) == EINVAL
    assert _norm(one, 1, norm=0) == _norm(one, 1, norm=4098) == _norm(one, 1, ws=0) == _norm(one, 1, ws=4096 + 16) == EINVAL
    assert _clip(one, 1, norm=0) == _clip(one, 1, limit=-1.0) == _clip(one, 1, limit=NAN) == EINVAL
    assert _norm(one, 1, bytes_=7) == EWORKSPACE
