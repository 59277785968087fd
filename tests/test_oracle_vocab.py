"""The 64-bit oracle of the vocabulary's losses against torch's own losses, autograd and differences (no GPU)."""
import pytest
import torch
import torch.nn.functional as F

from oracle import vocab_oracle as orc


def _inputs(N, M, V, K=0):
    g = torch.Generator().manual_seed(N * 1000 + V + K)
    x, w = torch.randn(N, M, generator=g).double(), torch.randn(V, M, generator=g).double() / M ** 0.5
    target = torch.randint(0, V, (N,), generator=g)
    idx = torch.randint(0, V, (N, max(K, 1)), generator=g)       # (repeated indices among them)
    logit = 2 * torch.randn(N, max(K, 1), generator=g)
    dloss = torch.rand(N, generator=g).double()
    return x, w, target, idx, logit, dloss


@pytest.mark.parametrize("N,M,V", [(1, 8, 1), (5, 16, 9), (40, 24, 101)])
def test_cross_entropy_is_torchs(N, M, V):
    x, w, target, _, _, dloss = _inputs(N, M, V)
    target[::3] = -1
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    want = F.cross_entropy(xg @ wg.t(), target, ignore_index=-1, reduction="none")
    loss, lse = orc.cross_entropy(x, w, target)
    assert torch.allclose(loss, want, atol=1e-13, rtol=1e-12)
    assert torch.allclose(lse[target >= 0], torch.logsumexp(x @ w.t(), 1)[target >= 0]) and (lse[target < 0] == 0).all()
    (want * dloss).sum().backward()
    q, has = orc.target_weights(N, V, target, x.device)
    dx, dw, _ = orc.backward(x, w, dloss, q, has)
    assert torch.allclose(dx, xg.grad, atol=1e-13) and torch.allclose(dw, wg.grad, atol=1e-13)


@pytest.mark.parametrize("N,M,V,K,T", [(1, 8, 4, 1, 1.0), (30, 16, 50, 7, 2.5), (9, 8, 3, 12, 0.5)])
def test_distillation_is_the_divergence(N, M, V, K, T):
    x, w, _, idx, logit, dloss = _inputs(N, M, V, K)
    if N > 1:
        idx[1], logit[2], idx[3, K // 2:] = -1, -torch.inf, V + 3
    q, has, _, _ = orc.teacher_weights(N, V, idx, logit, T, x.device)
    assert torch.allclose(q.sum(1), has.double())
    # loss = sum over entries of q log q minus sum over the vocabulary of q log p: with every index once, the KL divergence
    once = torch.tensor([len(set(r.tolist()) - {-1, V + 3}) == int(((r >= 0) & (r < V)).sum()) for r in idx])
    logp = F.log_softmax(x @ w.t() / T, 1)
    kl = F.kl_div(logp, q, reduction="none").sum(1)
    loss, _, ze = orc.distill(x, w, idx, logit, T)
    assert torch.allclose(loss[once & has], kl[once & has], atol=1e-12) and (loss[~has] == 0).all()
    assert torch.equal(ze == 0, ~((idx >= 0) & (idx < V) & (logit != -torch.inf)))
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    (-(q * F.log_softmax(xg @ wg.t() / T, 1)).sum(1) * dloss).sum().backward()
    dx, dw, _ = orc.backward(x, w, dloss, q, has, T)
    assert torch.allclose(dx, xg.grad, atol=1e-12) and torch.allclose(dw, wg.grad, atol=1e-12)


def test_gradients_by_differences():
    N, M, V, K, T = 6, 8, 11, 4, 1.7
    x, w, _, idx, logit, dloss = _inputs(N, M, V, K)
    idx[2] = -1
    q, has, _, _ = orc.teacher_weights(N, V, idx, logit, T, x.device)
    dx, dw, _ = orc.backward(x, w, dloss, q, has, T)
    f = lambda x, w: (orc.distill(x, w, idx, logit, T)[0] * dloss).sum()
    h = 1e-6
    for t, grad in ((x, dx), (w, dw)):
        for i in range(0, t.numel(), 7):
            e = torch.zeros_like(t)
            e.view(-1)[i] = h
            up = f(x + e, w) - f(x - e, w) if t is x else f(x, w + e) - f(x, w - e)
            assert abs(up / (2 * h) - grad.view(-1)[i]) < 1e-8
