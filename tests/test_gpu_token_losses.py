"""Preference and policy losses on token losses, and their gradients, against the formulas in 64 bits and against differences.

u = 2^-24.  Sums and pair losses are formed in 64 bits and rounded once (u), functions of a pair in 64 bits too; the backward pass
starts from the ratios as they are stored.  Policy, per token: r = exp(lr) with lr rounded to fp32 (|lr| u) and an exponential good to 2 u; products and
sums three roundings; x = nll - ref is rounded once: e^x - 1 - x then by |e^x - 1| |x| u, its series (|x| < 1) by 12 u relative, the difference beyond by
(e^x + 1 + |x|) 2 u; e^x - 1 by e^x |x| u and 2 u."""
import math

import pytest
import torch

import paper_2006_16668_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
V = 1000


def nan(*s):
    return torch.full(s, float("nan"), device=DEV)


def tokens(G, S, g, empty=0.3):
    """Token losses (NaN and infinity where there is no target), a reference's, targets."""
    old = 2 * torch.randn(G, S, generator=g, device=DEV).abs() + 1e-3
    nll = (old + 0.3 * torch.randn(G, S, generator=g, device=DEV)).clamp_(min=0)
    target = torch.randint(0, V, (G, S), generator=g, device=DEV, dtype=torch.int32)
    none = torch.rand(G, S, generator=g, device=DEV) < empty
    target = torch.where(none, torch.where(torch.rand(G, S, generator=g, device=DEV) < 0.5, -1, V), target.long()).int()
    nll[none] = float("nan")
    old[none] = float("inf")
    return nll, old, target


def pref_reference(ratio, kind, beta, e, dloss=None):
    h = ratio[0::2] - ratio[1::2]
    sp = lambda x: torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))
    sig = torch.sigmoid
    if kind == "logistic":
        loss = (1 - e) * sp(-beta * h) + e * sp(beta * h)
        dh = beta * (e * sig(beta * h) - (1 - e) * sig(-beta * h))
        size = beta * (e * sig(beta * h) + (1 - e) * sig(-beta * h))
    else:
        loss, dh = (h - 0.5 / beta) ** 2, 2 * (h - 0.5 / beta)
        size = dh.abs()
    return loss, (dh, size)


def starts(kind, P, N, g):
    if kind == "even":
        return [i * (N // (2 * P)) for i in range(2 * P + 1)]
    if kind == "empty":                                          # no sequence has a token
        return [N // 2] * (2 * P + 1)
    if kind == "outside":                                        # edges before the first and past the last token
        cuts = [-7] + [i * N // (2 * P) for i in range(1, 2 * P)] + [N + 9]
        return cuts
    cuts = sorted(torch.randint(0, N + 1, (2 * P + 1,), generator=g, device=DEV).tolist())
    return cuts


@pytest.mark.parametrize("loss_kind,beta,e", [("logistic", 0.1, 0.0), ("logistic", 0.7, 0.2), ("squared", 0.2, 0.0)])
@pytest.mark.parametrize("P,G,S,kind", [(1, 1, 1, "even"), (1, 2, 1, "even"), (3, 6, 41, "even"), (5, 1, 777, "any"), (2, 7, 300, "outside"), (4, 3, 33, "empty"),
                                        (200, 1, 403, "any"), (1, 1, 40001, "any"), (2100, 2100, 5, "any"), (64, 128, 512, "even")])
def test_preference(P, G, S, kind, loss_kind, beta, e):
    g = torch.Generator(device=DEV).manual_seed(P * 3 + S)
    N = G * S
    nll, ref, target = tokens(G, S, g)
    edges = starts(kind, P, N, g)
    start = torch.tensor(edges, dtype=torch.int32, device=DEV)
    sh, dims = moe.MoEShape(G, S, 8, 8, 2, 1, "f32"), moe.PreferenceDims(P, V, beta, e, loss_kind)
    loss, ratio, dnll = nan(P), nan(2 * P), nan(G, S)
    moe.moe_preference_loss(sh, dims, nll, ref, target, start, loss, ratio)
    counts = ((target >= 0) & (target < V)).view(-1)
    diff = torch.where(counts, ref.double().view(-1) - nll.double().view(-1), 0.0)
    total = torch.cat([torch.zeros(1, device=DEV, dtype=torch.float64), diff.cumsum(0)])
    cut = start.long().clamp(0, N)
    want = total[cut[1:]] - total[cut[:-1]]
    assert ((ratio.double() - want).abs() <= U * want.abs() + 1e-9).all()
    l, _ = pref_reference(want, loss_kind, beta, e)
    # 1e-9 in h (the oracle's running sum): as much again times the slope of the loss
    slope = pref_reference(want, loss_kind, beta, e)[1][1]
    assert ((loss.double() - l).abs() <= 2 * U * l.abs() + 4e-9 * (1 + slope)).all()
    dloss = torch.rand(P, generator=g, device=DEV) + 0.5
    moe.moe_preference_loss_backward(sh, dims, target, start, ratio, dloss, dnll)
    dh, size = pref_reference(ratio.double(), loss_kind, beta, e)[1]
    per = torch.stack([-dh * dloss, dh * dloss], 1).view(-1)
    err = torch.stack([size * dloss] * 2, 1).view(-1)
    seq = torch.searchsorted(start.long(), torch.arange(N, device=DEV), right=True) - 1
    inside = (seq >= 0) & (seq < 2 * P) & counts
    seq = seq.clamp(0, 2 * P - 1)
    want = torch.where(inside, per[seq], 0.0).view(G, S)
    assert ((dnll.double() - want).abs() <= torch.where(inside, err[seq], 0.0).view(G, S) * (U + 1e-12)).all()
    again = nan(G, S)
    moe.moe_preference_loss_backward(sh, dims, target, start, ratio, dloss, again)
    assert torch.equal(again, dnll)


@pytest.mark.parametrize("h", [-2e4, -700.0, -40.0, -1e-6, 0.0, 3e-5, 40.0, 700.0, 3e4])
def test_preference_of_sure_pairs(h):
    """A margin of any size: the loss keeps its own digits, and nothing overflows."""
    sh, dims = moe.MoEShape(2, 1, 8, 8, 2, 1, "f32"), moe.PreferenceDims(1, V, 1.0)
    nll, ref = torch.tensor([[0.0], [max(h, 0.0)]], device=DEV), torch.tensor([[max(h, 0.0)], [max(h, 0.0)]], device=DEV)
    if h < 0:
        nll, ref = torch.tensor([[-h], [0.0]], device=DEV), torch.tensor([[0.0], [0.0]], device=DEV)
    h = float((ref[0, 0].double() - nll[0, 0].double()) - (ref[1, 0].double() - nll[1, 0].double()))
    target, start = torch.zeros(2, 1, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    loss, ratio, dnll = nan(1), nan(2), nan(2, 1)
    moe.moe_preference_loss(sh, dims, nll, ref, target, start, loss, ratio)
    moe.moe_preference_loss_backward(sh, dims, target, start, ratio, torch.ones(1, device=DEV), dnll)
    want = math.log1p(math.exp(-abs(h))) + max(-h, 0.0)
    slope = -1 / (1 + math.exp(h)) if h < 500 else -math.exp(-h)
    assert abs(float(loss) - want) <= 2 * U * want + 1e-45
    assert abs(float(dnll[1]) - slope) <= 2 * U * abs(slope) + 1e-45 and float(dnll[0]) == -float(dnll[1])


def policy_reference(nll, old, ref, adv, low, high, beta):
    lr = old.double() - nll.double()
    a = adv.double() if adv.dim() == 2 else adv.double()[:, None]
    r = lr.exp()
    up, down = (a > 0) & (r > 1 + high), (a < 0) & (r < 1 - low)
    bounded = torch.where(up, 1 + high, torch.where(down, 1 - low, r))
    loss = torch.where(a == 0, 0.0, -a * bounded)
    grad = torch.where(up | down | (a == 0), 0.0, a * r)
    e_r = r * (lr.abs() + 2) * U
    e_loss, e_grad = a.abs() * torch.where(up | down, 2 * U, e_r) + 3 * U * loss.abs(), a.abs() * e_r + 3 * U * grad.abs()
    kl = torch.zeros_like(loss)
    if ref is not None:
        x = nll.double() - ref.double()
        kl = torch.expm1(x) - x
        e_kl = torch.expm1(x).abs() * x.abs() * U + torch.where(x.abs() < 1.001, 12 * U * kl, (x.exp() + 1 + x.abs()) * 2 * U)
        loss, e_loss = loss + beta * kl, e_loss + beta * (e_kl + 3 * U * kl) + U * (loss + beta * kl).abs()
        grad = grad + beta * torch.expm1(x)
        e_grad = e_grad + beta * (x.exp() * x.abs() + 4 * torch.expm1(x).abs()) * U + U * grad.abs()
    else:
        e_kl = torch.zeros_like(kl)
    return (loss, e_loss), (kl, e_kl), (grad, e_grad)


@pytest.mark.parametrize("G,S", [(1, 1), (1, 3), (3, 1), (5, 7), (2, 1021), (1000, 1), (37, 100), (513, 333)])
@pytest.mark.parametrize("per_token,beta,low,high", [(True, 0.04, 0.2, 0.2), (False, 0.0, 0.2, 0.28), (False, 0.5, 0.0, 0.0), (True, 0.1, 1.0, 3.0)])
def test_policy(G, S, per_token, beta, low, high):
    g = torch.Generator(device=DEV).manual_seed(G * 5 + S)
    nll, old, target = tokens(G, S, g)
    ref = nll + 0.5 * torch.randn(G, S, generator=g, device=DEV) if beta else None
    adv = torch.randn(*((G, S) if per_token else (G,)), generator=g, device=DEV)
    adv.view(-1)[::5] = 0.0
    counts = (target >= 0) & (target < V)
    if per_token:
        adv[~counts] = float("nan")
    sh, dims = moe.MoEShape(G, S, 8, 8, 2, 1, "f32"), moe.PolicyDims(V, low, high, beta)
    loss, kl, dnll, dloss = nan(G, S), nan(G, S), nan(G, S), torch.rand(G, S, generator=g, device=DEV) + 0.5
    dloss[~counts] = float("inf")
    moe.moe_policy_loss(sh, dims, nll, old, ref, adv, target, loss, kl)
    moe.moe_policy_loss_backward(sh, dims, nll, old, ref, adv, target, dloss, dnll)
    (l, e_l), (k, e_k), (d, e_d) = policy_reference(nll, old, ref, adv, low, high, beta)
    for got, want, err in ((loss, l, e_l), (kl, k, e_k), (dnll, d * dloss, (e_d + U * d.abs()) * dloss)):
        assert (got[~counts] == 0).all()
        assert ((got.double() - want).abs() <= err + 1e-40)[counts].all()
    bare = nan(G, S)
    moe.moe_policy_loss(sh, dims, nll, old, ref, adv, target, bare)
    assert torch.equal(bare, loss)
    assert (kl[counts] >= 0).all()


def test_policy_at_the_bound_and_far_from_it():
    """Ratios one step of fp32 on either side of a bound, at it, and where the exponential overflows or vanishes."""
    high = math.exp(0.25) - 1                                    # the bound lies at a log-ratio of 0.25, to 64 bits
    lr = torch.tensor([0.25 - 2.0 ** -20, 0.25 + 2.0 ** -20, 100.0, 100.0, -200.0, -200.0, 0.0], device=DEV)
    adv = torch.tensor([1.0, 1.0, 2.0, -2.0, 2.0, -2.0, 0.0], device=DEV)
    n = lr.numel()
    old, nll = torch.full((n, 1), 1.0, device=DEV) + lr.view(n, 1).clamp(min=0), torch.full((n, 1), 1.0, device=DEV) - lr.view(n, 1).clamp(max=0)
    target = torch.zeros(n, 1, dtype=torch.int32, device=DEV)
    sh, dims = moe.MoEShape(n, 1, 8, 8, 2, 1, "f32"), moe.PolicyDims(V, 0.2, high)
    loss, dnll = nan(n, 1), nan(n, 1)
    moe.moe_policy_loss(sh, dims, nll, old, None, adv, target, loss)
    moe.moe_policy_loss_backward(sh, dims, nll, old, None, adv, target, torch.ones(n, 1, device=DEV), dnll)
    got, up = loss.view(-1).tolist(), dnll.view(-1).tolist()
    r = math.exp(0.25 - 2.0 ** -20)
    assert abs(got[0] + r) <= 4 * U * r and abs(up[0] - r) <= 4 * U * r
    assert abs(got[1] + 1 + high) <= 4 * U and up[1] == 0
    assert abs(got[2] + 2 * (1 + high)) <= 8 * U and up[2] == 0
    assert got[3] == float("inf") and up[3] == -float("inf")      # exp(100) is past fp32, and nothing bounds it there
    assert got[4] == 0 and up[4] == 0
    assert abs(got[5] - 1.6) <= 4 * U and up[5] == 0
    assert got[6] == 0 and up[6] == 0


def test_losses_against_differences():
    """d loss / d nll by the calls' own values in steps that fp32 resolves."""
    g = torch.Generator(device=DEV).manual_seed(1)
    G, S, P = 4, 6, 2
    nll = torch.rand(G, S, generator=g, device=DEV) + 1
    ref, old = nll + 0.2 * torch.rand(G, S, generator=g, device=DEV), nll + 0.05
    target = torch.zeros(G, S, dtype=torch.int32, device=DEV)
    start = torch.arange(0, G * S + 1, S, dtype=torch.int32, device=DEV)
    sh, pd, qd = moe.MoEShape(G, S, 8, 8, 2, 1, "f32"), moe.PreferenceDims(P, V, 0.9, 0.1), moe.PolicyDims(V, 0.2, 0.2, 0.3)
    adv = torch.randn(G, S, generator=g, device=DEV)

    def pref(x):
        loss, ratio = nan(P), nan(2 * P)
        moe.moe_preference_loss(sh, pd, x, ref, target, start, loss, ratio)
        return loss.double().sum().item(), ratio

    def pol(x):
        loss = nan(G, S)
        moe.moe_policy_loss(sh, qd, x, old, ref, adv, target, loss)
        return loss.double().sum().item()

    dp, dq = nan(G, S), nan(G, S)
    moe.moe_preference_loss_backward(sh, pd, target, start, pref(nll)[1], torch.ones(P, device=DEV), dp)
    moe.moe_policy_loss_backward(sh, qd, nll, old, ref, adv, target, torch.ones(G, S, device=DEV), dq)
    step = 2.0 ** -7                                             # error: its square, and 4 u / step of the values
    for i, j in ((0, 0), (1, 3), (2, 5), (3, 2)):
        up, down = nll.clone(), nll.clone()
        up[i, j] += step
        down[i, j] -= step
        assert math.isclose((pref(up)[0] - pref(down)[0]) / (2 * step), float(dp[i, j]), rel_tol=1e-3, abs_tol=2e-4)
        assert math.isclose((pol(up) - pol(down)) / (2 * step), float(dq[i, j]), rel_tol=1e-3, abs_tol=1e-3)


def test_nothing_is_written_outside():
    """Outputs in the middle of buffers, sizes that end inside a thread's four."""
    g = torch.Generator(device=DEV).manual_seed(2)
    G, S = 3, 67
    nll, old, target = tokens(G, S, g)
    buf = torch.full((3, 1024), 7.0, device=DEV)
    at = [b[256:256 + G * S].view(G, S) for b in buf]
    sh = moe.MoEShape(G, S, 8, 8, 2, 1, "f32")
    adv = torch.randn(G, generator=g, device=DEV)
    moe.moe_policy_loss(sh, moe.PolicyDims(V), nll, old, None, adv, target, at[0])
    moe.moe_policy_loss_backward(sh, moe.PolicyDims(V), nll, old, None, adv, target, torch.ones(G, S, device=DEV), at[1])
    start = torch.tensor([0, 50, 150], dtype=torch.int32, device=DEV)
    moe.moe_preference_loss_backward(sh, moe.PreferenceDims(1, V, 0.1), target, start, torch.zeros(2, device=DEV), torch.ones(1, device=DEV), at[2])
    for b in buf:
        assert (b[:256] == 7).all() and (b[256 + G * S:] == 7).all() and torch.isfinite(b).all()
    assert (at[2].view(-1)[150:] == 0).all()
