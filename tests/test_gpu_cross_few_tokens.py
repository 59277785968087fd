"""Calls of few tokens, the steps of generation among them: nothing that a whole head's result hangs on is rounded to bf16 once.

q, the probabilities and ctx, and in the backward pass dctx and dS, are pairs of bf16: the second is what the first leaves, rounded, 2^-16 of the number.  With u = 2^-24, h = 2^-8 and core()'s bounds in
fp32 (sums, exponentials), q is off by 2^-16 |q| + M u |u|.|wq|, ctx by 2^-16 (sum p |v| + |ctx|) more, and the result by its own rounding."""
import pytest
import torch

import paper_2006_16668_amd as moe
from cross_bounds import DT, HALF, U, assert_within, core
from test_gpu_cross_attention import DEV, _rand, held, lens, selection

pytestmark = pytest.mark.gpu
PAIR = 2.0 ** -16

# B, Lq, Lk, M, heads, kv_heads, d, lengths
CASES = [(1, 1, 55, 200, 1, 1, 64, None), (1, 4, 385, 848, 2, 2, 128, None), (2, 1, 426, 440, 4, 1, 64, None), (1, 1, 794, 1440, 32, 8, 64, None),
         (1, 4, 53, 1024, 16, 16, 128, None), (64, 1, 300, 1024, 16, 16, 128, "any"), (6, 2, 1, 64, 1, 1, 64, "ends"), (6, 3, 64, 256, 2, 1, 128, "ends"),
         (6, 5, 65, 264, 8, 2, 64, "ends"), (1, 16, 700, 512, 4, 4, 64, None), (1, 17, 129, 512, 4, 4, 128, None), (3, 31, 190, 72, 2, 2, 64, "any"),
         (1, 65, 333, 512, 4, 4, 64, "any"), (2, 33, 1000, 256, 16, 1, 64, "any"), (1, 128, 260, 1024, 4, 4, 128, None), (3, 1, 8200, 136, 2, 2, 64, "any"),
         (5, 2, 4100, 520, 16, 2, 128, "any"), (2, 48, 757, 512, 8, 2, 64, "any"), (1, 30, 344, 256, 1, 1, 128, None), (7, 18, 765, 512, 4, 1, 64, "ends")]


def inputs(c, seed=0, scale=1.5):
    B, Lq, Lk, M, heads, kv_heads, d, kind = c
    g = torch.Generator(device=DEV).manual_seed(seed + B + Lq + Lk + M)
    A, W, bf = heads * d, 2 * kv_heads * d, torch.bfloat16
    u, kv = _rand(g, B, Lq, M, dt=bf), _rand(g, B, Lk, W, dt=bf)
    wq, wo = (scale * torch.randn(M, A, generator=g, device=DEV) / M ** 0.5).to(bf), (torch.randn(A, M, generator=g, device=DEV) / A ** 0.5).to(bf)
    src_len = lens(B, Lk, kind, g)
    n = held(src_len, B, Lk)
    for b in range(B):
        kv[b, n[b]:] = float("nan")
    return moe.MoEShape(B, Lq, M, 64, 2, 1), moe.CrossDims(B, Lq, Lk, heads, d, kv_heads), u, kv, src_len, n, wq, wo


def call(sh, dims, u, kv, src_len, wq, wo, train=False):
    out = torch.full_like(u, float("nan"))
    ws = torch.full(((moe.moe_cross_train_workspace_bytes if train else moe.moe_cross_workspace_bytes)(sh, dims),), 255, dtype=torch.uint8, device=DEV)
    (moe.moe_cross_attention_train if train else moe.moe_cross_attention)(sh, dims, u, kv, src_len, wq, wo, out, ws)
    return out


@pytest.mark.parametrize("c", CASES)
def test_results_carry_their_own_rounding_only(c):
    sh, dims, u, kv, src_len, n, wq, wo = inputs(c)
    print(f"case {c}", flush=True)
    out = call(sh, dims, u, kv, src_len, wq, wo)
    assert torch.equal(out, call(sh, dims, u, kv, src_len, wq, wo, train=True))
    M, A = sh.M, dims.heads * dims.d
    D = lambda t: t.double()
    q = D(u) @ D(wq)
    e_q = PAIR * q.abs() + 2 * M * U * (D(u).abs() @ D(wq).abs())
    share = dims.heads // dims.key_heads
    ctx, e_ctx = core(q, kv, n, dims.key_heads, share, dims.d, "f32", None, e_q)["ctx"]
    size, _ = core(q, kv.abs().where(torch.arange(2 * dims.key_heads * dims.d, device=DEV) >= dims.key_heads * dims.d, kv), n, dims.key_heads, share, dims.d, "f32")["ctx"]
    e_ctx = e_ctx + PAIR * (size + ctx.abs())                    # (size: sum p |v|)
    want = ctx @ D(wo)
    assert_within(out, want, e_ctx @ D(wo).abs() + 4 * A * U * (ctx.abs() @ D(wo).abs()) + HALF["bf16"] * want.abs(), "out")
    # rounding alone: an error of h / sqrt(3) of the power of two below a number, 0.4 h of numbers spread over a binade
    if want.numel() >= 400:
        err = float((D(out) - want).norm() / want.norm())
        assert err < 0.55 * HALF["bf16"], err / HALF["bf16"]


@pytest.mark.parametrize("c", [(1, 3, 70, 128, 2, 2, 64, None), (2, 3, 600, 128, 1, 1, 128, None), (1, 40, 130, 128, 2, 2, 64, None)])
def test_states_shut_out_by_an_infinite_key(c):
    """A key that makes a score of -inf for every query takes its state out, whatever the second terms make of it (0 times infinity)."""
    B, Lq, Lk, M, heads, kv_heads, d, _ = c
    g = torch.Generator(device=DEV).manual_seed(1)
    A, bf = heads * d, torch.bfloat16
    M = max(M, 2 * A)
    u, kv = _rand(g, B, Lq, M, dt=bf), _rand(g, B, Lk, 2 * A, dt=bf)
    u[..., 0:A:d] = 1.0 + torch.rand(B, Lq, heads, generator=g, device=DEV).to(bf)          # (q's first d is positive)
    sh, dims = moe.MoEShape(B, Lq, M, 64, 2, 1), moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    wq, wo = selection(M, A, bf), selection(A, M, bf)
    half = Lk // 2
    kv[:, half:, 0:A:d] = float("-inf")
    out = call(sh, dims, u, kv, None, wq, wo)
    src_len = torch.full((B,), half, dtype=torch.int32, device=DEV)
    want = call(sh, dims, u, kv, src_len, wq, wo)
    assert torch.isfinite(want).all()
    assert ((out.double() - want.double()).abs() <= 2 * HALF["bf16"] * want.double().abs() + 1e-6).all()


@pytest.mark.parametrize("value", [6e37, 1.0, 1e-36])
def test_large_and_small_values_pass(value):
    """Sums of five states stay below the end of fp32: the mean of equal values is that value, and products with 0 are 0."""
    B, Lq, Lk, d, M, bf = 1, 2, 5, 64, 128, torch.bfloat16
    sh, dims = moe.MoEShape(B, Lq, M, 64, 2, 1), moe.CrossDims(B, Lq, Lk, 1, d)
    u, kv = torch.zeros(B, Lq, M, dtype=bf, device=DEV), torch.zeros(B, Lk, 2 * d, dtype=bf, device=DEV)
    kv[..., d] = value
    out = call(sh, dims, u, kv, None, selection(M, d, bf), selection(d, M, bf))
    assert (out[..., 1:] == 0).all() and (out[..., 0] == kv[0, 0, d]).all()


@pytest.mark.parametrize("c", [CASES[4], CASES[5], CASES[8], CASES[15]])
def test_nothing_is_written_outside_and_what_the_workspace_held_does_not_count(c):
    sh, dims, u, kv, src_len, n, wq, wo = inputs(c)
    want = call(sh, dims, u, kv, src_len, wq, wo)
    for train, size in ((False, moe.moe_cross_workspace_bytes(sh, dims)), (True, moe.moe_cross_train_workspace_bytes(sh, dims))):
        for fill in (0, 0x3f, 255):
            ws = torch.full((size + 8192,), 77, dtype=torch.uint8, device=DEV)
            ws[4096:4096 + size] = fill
            room = torch.full((u.numel() + 1024,), 7.0, dtype=torch.bfloat16, device=DEV)
            out = room[512:512 + u.numel()].view_as(u)
            (moe.moe_cross_attention_train if train else moe.moe_cross_attention)(sh, dims, u, kv, src_len, wq, wo, out, ws[4096:4096 + size])
            assert torch.equal(out, want)
            assert (room[:512] == 7).all() and (room[-512:] == 7).all() and (ws[:4096] == 77).all() and (ws[-4096:] == 77).all()


def backward(c, seed=0, scale=1.5, select=False, fill=255):
    """Gradients by the calls, and q, dctx, and the attention's own gradients in 64 bits.  select: mem holds kv whole, so that dmem is dkv."""
    B, Lq, Lk, M, heads, kv_heads, d, _ = c
    sh, dims, u, kv, src_len, n, wq, wo = inputs(c, seed, scale)
    W, bf = 2 * kv_heads * d, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(seed + 77)
    dout = _rand(g, B, Lq, M, dt=bf)
    if select:
        assert W <= M
        wkv, mem = selection(M, W, bf), torch.zeros(B, Lk, M, dtype=bf, device=DEV)
        mem[..., :W] = kv
    else:
        wkv, mem = (torch.randn(M, W, generator=g, device=DEV) / M ** 0.5).to(bf), _rand(g, B, Lk, M, dt=bf)
        for b in range(B):
            mem[b, n[b]:] = float("inf")
    bytes_ = lambda size: torch.full((size,), fill, dtype=torch.uint8, device=DEV)
    out, fwd = torch.empty_like(u), bytes_(moe.moe_cross_train_workspace_bytes(sh, dims))
    moe.moe_cross_attention_train(sh, dims, u, kv, src_len, wq, wo, out, fwd)
    grads = {k: torch.full_like(t, float("nan")) for k, t in (("du", u), ("dmem", mem), ("dwq", wq), ("dwkv", wkv), ("dwo", wo))}
    moe.moe_cross_attention_backward(sh, dims, u, mem, kv, src_len, wq, wkv, wo, dout, fwd, grads, bytes_(moe.moe_cross_backward_workspace_bytes(sh, dims)))
    D = lambda t: t.double()
    q, dctx = D(u) @ D(wq), D(dout) @ D(wo).t()
    ref = core(q, kv, n, kv_heads, heads // kv_heads, d, "f32", dctx)
    flat = lambda t: t.reshape(-1, t.shape[-1])
    held_mem = D(torch.stack([torch.where(torch.arange(Lk, device=DEV)[:, None] < n[b], mem[b], 0.0) for b in range(B)]))
    want = {"du": ref["dq"][0] @ D(wq).t(), "dmem": ref["dkv"][0] @ D(wkv).t(), "dwq": flat(D(u)).t() @ flat(ref["dq"][0]),
            "dwkv": flat(held_mem).t() @ flat(ref["dkv"][0]), "dwo": flat(ref["ctx"][0]).t() @ flat(D(dout))}
    return grads, want, ref, n, (D(u), D(wq), D(dout), D(wo), dctx)


# besides: dK and dV in ranges of columns, two columns and many of them to a key head, one state
GRADIENT_CASES = CASES + [(1, 128, 100, 512, 8, 2, 64, None), (2, 48, 2000, 512, 8, 1, 64, "any"), (1, 128, 300, 1024, 8, 2, 128, "any"), (3, 9, 2, 264, 1, 1, 128, None),
                          (11, 1, 2, 136, 1, 1, 64, None), (64, 2, 40, 512, 4, 4, 128, "any"), (4, 32, 64, 72, 2, 2, 64, "ends")]


@pytest.mark.parametrize("c", GRADIENT_CASES)
def test_gradients_are_off_by_what_is_stored(c):
    """Between the inputs and a gradient lie a sum that is stored in bf16 (dq, dK and dV, ctx) and the result itself, 0.4 h each in norm of numbers spread over a
    binade, independent of one another: 0.6 h; 1 h where there are too few numbers for a mean.  What is a pair is off by 2^-16."""
    print(f"case {c}", flush=True)
    grads, want, ref, n, _ = backward(c)
    B, Lq, Lk, M, heads, kv_heads, d, _ = c
    for k, w in want.items():
        got = grads[k].double()
        assert torch.isfinite(got).all(), k
        if w.norm() < 1e-9 * got.numel() ** 0.5:                # (of one state nothing passes to q and K: what 64 bits leave)
            assert got.abs().max() <= 1e-9, k
            continue
        err = float((got - w).norm() / w.norm()) / HALF["bf16"]
        stored = min(B * Lq * heads, sum(n) * kv_heads) * d
        assert err < (0.75 if stored >= 1000 else 1.0), (k, err)
    for b in range(B):
        assert (grads["dmem"][b, n[b]:] == 0).all()
        if n[b] <= 1:
            assert (grads["du"][b] == 0).all()


@pytest.mark.parametrize("c", [c for c in GRADIENT_CASES if 2 * c[5] * c[6] <= c[3]])
def test_keys_and_values_gradients_element_by_element(c):
    """dK and dV as dmem shows them: core()'s bounds in fp32, with q and dctx off by 2^-16 and their sums' roundings, P and dS by 2^-16, the result by h."""
    print(f"case {c}", flush=True)
    grads, _, _, n, (u, wq, dout, wo, dctx) = backward(c, select=True)
    B, Lq, Lk, M, heads, kv_heads, d, _ = c
    sh, dims, _, kv, *_ = inputs(c)
    W, share = 2 * kv_heads * d, heads // kv_heads
    q = u @ wq
    e_q = PAIR * q.abs() + 2 * M * U * (u.abs() @ wq.abs())
    e_g = PAIR * dctx.abs() + 2 * M * U * (dout.abs() @ wo.abs().t())
    dkv, err = core(q, kv, n, kv_heads, share, d, "f32", dctx, e_q)["dkv"]
    # what dctx's error and those of P and dS add
    sizes = torch.zeros_like(dkv)
    Kd = kv_heads * d
    for b in range(B):
        if n[b] == 0:
            continue
        for k in range(kv_heads):
            cols = slice(k * share * d, (k + 1) * share * d)
            Q, G, E = (t[b][:, cols].reshape(-1, d) for t in (q, dctx, e_g))
            K, V = kv[b, :n[b], k * d:(k + 1) * d].double(), kv[b, :n[b], Kd + k * d:Kd + (k + 1) * d].double()
            p = torch.softmax(Q @ K.t() / d ** 0.5, 1)
            dp, e_dp = G.abs() @ V.abs().t(), E @ V.abs().t()
            ds = p * (dp + (p * dp).sum(1, keepdim=True)) / d ** 0.5
            e_ds = p * (e_dp + (p * e_dp).sum(1, keepdim=True)) / d ** 0.5 + 4 * PAIR * ds
            sizes[b, :n[b], k * d:(k + 1) * d] = e_ds.t() @ Q.abs() + 4 * PAIR * ds.t() @ Q.abs()
            sizes[b, :n[b], Kd + k * d:Kd + (k + 1) * d] = p.t() @ E + 4 * PAIR * p.t() @ G.abs()
    assert_within(grads["dmem"][..., :W], dkv, err + sizes + 1.01 * HALF["bf16"] * dkv.abs(), "dkv")


@pytest.mark.parametrize("c", [GRADIENT_CASES[5], GRADIENT_CASES[7], GRADIENT_CASES[-6], GRADIENT_CASES[-5]])
def test_gradients_repeat_whatever_the_workspaces_held(c):
    want = backward(c)[0]
    for fill in (0, 0x3f, 255):
        got = backward(c, fill=fill)[0]
        for k, t in want.items():
            assert torch.equal(got[k], t), k


@pytest.mark.parametrize("c", [(6, 3, 64, 256, 2, 1, 128, "ends"), (6, 3, 65, 256, 2, 2, 64, "ends"), (6, 2, 4100, 512, 2, 2, 64, "ends"), (6, 2, 4100, 512, 2, 1, 128, "ends"),
                               (7, 18, 765, 512, 4, 1, 64, "ends"), (6, 16, 500, 512, 2, 2, 128, "ends")])
def test_probabilities_add_up(c):
    """With scores of some hundred, what q loses in bf16 moves a probability by far more than a rounding: statistics and scores are of the same q, so that of one
    state p is 1 (dV is the sum of dctx over the tokens), and of all the probabilities add up to 1."""
    B, Lq, Lk, M, heads, kv_heads, d, _ = c
    grads, _, _, n, (u, wq, dout, wo, dctx) = backward(c, scale=30.0, select=True)
    h, W = HALF["bf16"], 2 * kv_heads * d
    split = lambda t: t.view(B, Lq, kv_heads, heads // kv_heads, d).sum((1, 3)).view(B, kv_heads * d)
    total, size, terms = split(dctx), split(dctx.abs()), split(dout.abs() @ wo.abs().t())
    dv = grads["dmem"].double()[..., W // 2:W]
    for b in range(B):
        if n[b] == 0:
            continue
        # dV rounded (h of each state's, whose magnitudes add up to no more than size), fp32 sums; an exponential of a score s is off by 4 s u: s below 2000
        assert ((dv[b, :n[b]].sum(0) - total[b]).abs() <= (h + 2 * PAIR + 8000 * U) * size[b] + 4 * M * U * terms[b] + 1e-12).all(), b
        if n[b] == 1:
            assert ((dv[b, 0] - total[b]).abs() <= h * total[b].abs() + (2 * PAIR + 8000 * U) * size[b] + 4 * M * U * terms[b] + 1e-12).all(), b
