"""A decoder's training step where the policy's bounds hold some of the ratios, in norm within a few roundings; sources with fewer states than a batch of more
than 4 GB of them."""
import math

import pytest
import torch

import paper_2006_16668_amd as moe
from cross_bounds import DT, HALF, U, assert_within, core
from test_gpu_cross_attention import selection
from test_gpu_decoder_step import DEV, Step, nan

pytestmark = pytest.mark.gpu


def leaves(s):
    leaf = lambda t: t.double().requires_grad_(True)
    return leaf(s.u), leaf(s.mem), {k: leaf(t) for k, t in s.w.items()}


def token_losses(s, u, mem, w):
    """nll [B,Lq] in 64 bits."""
    d, K, share = s.d, s.kv_heads, s.heads // s.kv_heads
    out = []
    for b in range(s.B):
        n = int(s.len[b])
        q = (u[b] @ w["wq"]).view(s.Lq, K, share, d)
        kv = (mem[b, :n] @ w["wkv"]).view(n, 2, K, d)
        p = torch.softmax(torch.stack([q[:, k, j] @ kv[:, 0, k].t() for k in range(K) for j in range(share)]) / d ** 0.5, -1)
        ctx = torch.cat([p[k * share + j] @ kv[:, 1, k] for k in range(K) for j in range(share)], 1)
        z = ctx @ w["wo"] @ w["wv"].t()
        out.append(torch.logsumexp(z, -1) - z.gather(-1, s.target[b].clamp(min=0).long()[:, None])[:, 0])
    return torch.stack(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_policy_step_with_ratios_at_their_bounds(dtype):
    """Log-ratios of -0.6, -0.1, 0.1 and 0.6 against bounds at log 0.8 = -0.22 and log 1.2 = 0.18: none is nearer than 0.08 to one, which no rounding of
    nll (some 0.01) passes.  Ten stored intermediates lie between the inputs and a gradient, off by up to h of an element and 0.4 h in the mean; independent of one
    another they leave 1.3 h, and scores and losses of a few units make some three times that of it: 6 h.  (fp32: sums of a few hundred terms instead.)"""
    s = Step(dtype, "policy", seed=3)
    low = high = 0.2
    beta = 0.1
    s.qd = moe.PolicyDims(s.V, low, high, beta)
    u, mem, w = leaves(s)
    nll = token_losses(s, u, mem, w)
    g = torch.Generator(device=DEV).manual_seed(11)
    lr = torch.tensor([-0.6, -0.1, 0.1, 0.6], device=DEV)[torch.randint(0, 4, (s.B, s.Lq), generator=g, device=DEV)]
    s.ref = (nll.detach() + lr).float()
    has, a = s.target >= 0, s.adv.double()[:, None]
    r = torch.exp(s.ref.double() - nll)
    held = ((a > 0) & (r > 1 + high)) | ((a < 0) & (r < 1 - low))
    x = nll - s.ref.double()
    bounded = torch.where(held, torch.where(a > 0, 1 + high, 1 - low), r)
    loss = torch.where(has, -a * bounded + beta * (torch.expm1(x) - x), 0.0)
    (loss * s.up).sum().backward()
    counts = held & has
    assert (counts & (a > 0)).any() and (counts & (a < 0)).any() and (has & ~held).any()
    grads = {f"d{k}": t.grad for k, t in w.items()}
    norm = math.sqrt(sum(float((t ** 2).sum()) for t in grads.values()))
    scale = min(1.0, s.max_norm / norm)
    assert scale < 1
    got = s.run()
    torch.cuda.synchronize()
    tol = 6 * HALF["bf16"] if dtype == "bf16" else 800 * U
    for k, want in {"loss": loss.detach(), "norm": torch.tensor([norm], device=DEV, dtype=torch.float64), "du": u.grad, "dmem": mem.grad,
                    **{k: t * scale for k, t in grads.items()}}.items():
        err = float((got[k].double() - want).norm() / want.norm())
        assert err < tol, (k, err / tol)
    # the gradient at nll itself: of a token that is held, only the KL term's is left
    only = torch.where(counts, beta * torch.expm1(x.detach()) * s.up, 0.0)
    at = got["dnll"].double()[counts]
    assert ((at - only[counts]).abs() <= (0.02 if dtype == "bf16" else 1e-5) * beta * s.up.double()[counts] * 2).all()


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_a_step_in_bf16_within_a_few_roundings(kind):
    s = Step("bf16", kind, seed=5)
    got, want = s.run(), s.reference()
    torch.cuda.synchronize()
    for k, w in want.items():
        err = float((got[k].double() - w).norm() / w.norm())
        assert err < 6 * HALF["bf16"], (k, err / HALF["bf16"])


@pytest.mark.parametrize("dtype,Lq,Lk,lens", [("bf16", 3, 300_033, (299_001, 300_000)), ("bf16", 130, 300_033, (150_001, 297_777)), ("f32", 33, 270_001, (269_000,))])
def test_sources_that_end_past_4_gb(dtype, Lq, Lk, lens):
    """As test_states_past_4_gb, but sources end before the batch does: what stands behind them is NaN, the last 64 states before alone count, and the
    gradient of wkv is theirs."""
    g = torch.Generator(device=DEV).manual_seed(9)
    B, heads, d, dt = len(lens), 16, 128, DT[dtype]
    A = heads * d
    M, tail = 2 * A, 64
    print(f"case {dtype} {Lq} {Lk} {lens}", flush=True)
    dims, sh = moe.CrossDims(B, Lq, Lk, heads, d), moe.MoEShape(B, Lq, M, 64, 2, 1, dtype)
    u = torch.randn(B, Lq, M, generator=g, device=DEV).to(dt)
    u[..., 0:A:d] = 100.0
    kv = torch.zeros(B, Lk, 2 * A, dtype=dt, device=DEV)
    assert kv.numel() * kv.element_size() > 1 << 32
    kv[..., 0:A:d] = -40.0
    for b, n in enumerate(lens):
        kv[b, n - tail:n] = torch.randn(tail, 2 * A, generator=g, device=DEV).to(dt)
        kv[b, n - tail:n, 0:A:d] = 0.0
        kv[b, n:] = float("nan")
    last = torch.stack([kv[b, n - tail:n] for b, n in enumerate(lens)])
    src_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    wq, wkv, wo = selection(M, A, dt), selection(M, 2 * A, dt), selection(A, M, dt)
    u8 = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    out, fwd = nan(B, Lq, M, dt=dt), u8(moe.moe_cross_train_workspace_bytes(sh, dims))
    moe.moe_cross_attention_train(sh, dims, u, kv, src_len, wq, wo, out, fwd)
    dout = torch.randn(B, Lq, M, generator=g, device=DEV).to(dt)
    ref = core(u[..., :A], last, [tail] * B, heads, 1, d, dtype, dout[..., :A])
    extra = 1 + 64 * U / HALF[dtype]                             # (sums in ranges of states add as many roundings as there are ranges)
    assert_within(out[..., :A], ref["ctx"][0], extra * ref["ctx"][1], "ctx")
    grads = {"du": nan(B, Lq, M, dt=dt), "dmem": nan(B, Lk, M, dt=dt), "dwq": nan(M, A, dt=dt), "dwkv": nan(M, 2 * A, dt=dt), "dwo": nan(A, M, dt=dt)}
    moe.moe_cross_attention_backward(sh, dims, u, kv, kv, src_len, wq, wkv, wo, dout, fwd, grads, u8(moe.moe_cross_backward_workspace_bytes(sh, dims)))
    dkv, e_dkv = ref["dkv"]
    assert_within(grads["du"][..., :A], ref["dq"][0], extra * ref["dq"][1], "dq")
    for b, n in enumerate(lens):
        assert_within(grads["dmem"][b, n - tail:n], dkv[b], extra * e_dkv[b], "dkv")
        assert (grads["dmem"][b, :n - tail] == 0).all() and (grads["dmem"][b, n:] == 0).all()
    X, Y, E = last.double().view(B * tail, M), dkv.view(B * tail, -1), e_dkv.view(B * tail, -1)
    want = X.t() @ Y
    # rows of zeros add nothing, not even a rounding: sums of B tail terms, and h of the result
    assert_within(grads["dwkv"], want, extra * (X.abs().t() @ E) + 2 * B * tail * U * (X.abs().t() @ Y.abs()) + HALF[dtype] * want.abs(), "dwkv")
