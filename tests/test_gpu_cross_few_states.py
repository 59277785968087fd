"""Sources with few states in a batch of longer ones: their gradients are formed from their own states, whatever the others hold."""
import pytest
import torch

import paper_2006_16668_amd as moe
from cross_bounds import DT, HALF, assert_within, core
from test_gpu_cross_attention import DEV, _rand, run, selection

pytestmark = pytest.mark.gpu


# dq by blocks of 32 columns (B 4) and of 128 (B 40, more blocks of 32 than the units take)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,heads,kv_heads", [(4, 2, 2), (4, 4, 1), (40, 8, 8)])
@pytest.mark.parametrize("n", [1, 2, 3, 31, 32, 33, 63, 64])
def test_gradients_of_few_states_in_a_longer_batch(n, B, heads, kv_heads, d, dtype):
    """As for a batch of that many states: dq in norm is off by the roundings of dS and of itself, a third of h each in the mean, not by that of a
    stored ctx; of one state nothing passes to the query, to the last bit."""
    g = torch.Generator(device=DEV).manual_seed(n + B)
    Lq, Lk, dt, A, W = 65, 130, DT[dtype], heads * d, 2 * kv_heads * d
    M = max(A, W)
    print(f"case {n} {B} {heads} {kv_heads} {d} {dtype}", flush=True)
    u, kv, dout = (_rand(g, B, s, w, dt=dt) for s, w in ((Lq, M), (Lk, W), (Lq, M)))
    held = [Lk if b % 4 == 1 else n for b in range(B)]
    mem = torch.zeros(B, Lk, M, dtype=dt, device=DEV)
    mem[..., :W] = kv
    for b in range(B):
        kv[b, held[b]:] = float("nan")
        mem[b, held[b]:] = float("inf")
    src_len = torch.tensor(held, dtype=torch.int32, device=DEV)
    dims = moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    out, grads = run(dims, dtype, u, mem, kv, src_len, selection(M, A, dt), selection(M, W, dt), selection(A, M, dt), dout)
    ref = core(u[..., :A], kv, held, kv_heads, heads // kv_heads, d, dtype, dout[..., :A])
    assert_within(grads["du"][..., :A], *ref["dq"], "dq")
    assert_within(grads["dmem"][..., :W], *ref["dkv"], "dkv")
    few = [b for b in range(B) if held[b] == n]
    got, want = grads["du"][few][..., :A].double(), ref["dq"][0][few]
    if n == 1:
        assert (got == 0).all()
    else:
        err = (got - want).norm() / want.norm()
        assert err < (0.85 if dtype == "bf16" else 12) * HALF[dtype], float(err / HALF[dtype])


@pytest.mark.parametrize("n", [1, 2, 33, 64])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,heads", [(3, 2), (40, 8)])
def test_padding_changes_no_bits_of_dq(n, d, B, heads):
    """The same sources, padded to as many states as they hold at most and to more."""
    g = torch.Generator(device=DEV).manual_seed(n)
    Lq, A, dt = 65, heads * d, torch.bfloat16
    M, got = 2 * A, []
    u, kv, dout = (_rand(g, B, s, M, dt=dt) for s in (Lq, 64, Lq))
    src_len = torch.full((B,), n, dtype=torch.int32, device=DEV)
    for Lk in (64, 65, 200):
        more = torch.zeros(B, Lk, M, dtype=dt, device=DEV)
        more[:, :64] = kv
        # (the forward pass's form may depend on the padding: its ctx has no part in these gradients, its statistics in dK and dV only)
        _, grads = run(moe.CrossDims(B, Lq, Lk, heads, d), "bf16", u, more, more, src_len, selection(M, A, dt), selection(M, M, dt), selection(A, M, dt), dout)
        got.append(grads["du"])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
