"""Loss over a vocabulary and its gradients in 64 bits, from the formulas, for tokens without a target and teachers' lists with
gaps as well.  Torch tensors, so that large checks can run where the inputs are; no code of the library.

x [N,M], w [V,M]; cross entropy: target [N]; distillation: idx and logit [N,K], temperature T.
"""
import torch


def logits(x, w):
    return x.double() @ w.double().t()


def target_weights(N, V, target, device):
    """q [N,V]: what the softmax is compared with, and which rows have anything."""
    q = torch.zeros(N, V, dtype=torch.float64, device=device)
    has = (target >= 0) & (target < V)
    rows = torch.nonzero(has).view(-1)
    q[rows, target[rows].long()] = 1.0
    return q, has


def teacher_weights(N, V, idx, logit, T, device):
    there = (idx >= 0) & (idx < V) & (logit != -torch.inf)
    has = there.any(1)
    a = torch.where(there, logit.double(), -torch.inf)
    a = (a - torch.where(has, a.max(1).values, 0.0)[:, None]) / T
    e = torch.where(there, torch.exp(a), 0.0)
    qk = e / torch.where(has, e.sum(1), 1.0)[:, None]
    q = torch.zeros(N, V, dtype=torch.float64, device=device)
    for k in range(idx.shape[1]):                                # entries with one index add up
        rows = torch.nonzero(there[:, k]).view(-1)
        q[rows, idx[rows, k].long()] += qk[rows, k]
    return q, has, qk, there


def cross_entropy(x, w, target):
    """loss, lse [N]: 0 without a target."""
    z = logits(x, w)
    q, has = target_weights(z.shape[0], z.shape[1], target, x.device)
    lse = torch.logsumexp(z, 1)
    zt = torch.gather(z, 1, torch.where(has, target, 0).long()[:, None])[:, 0]
    return torch.where(has, lse - zt, 0.0), torch.where(has, lse, 0.0)


def distill(x, w, idx, logit, T):
    """loss, lse [N] and the logits at the entries [N,K]: 0 where there is none."""
    z = logits(x, w)
    _, has, qk, there = teacher_weights(z.shape[0], z.shape[1], idx, logit, T, x.device)
    lse = torch.logsumexp(z / T, 1)
    ze = torch.where(there, torch.gather(z, 1, torch.where(there, idx, 0).long()), 0.0)
    terms = torch.where(qk > 0, qk * (torch.log(qk) - ze / T + lse[:, None]), 0.0)
    return torch.where(has, terms.sum(1), 0.0), torch.where(has, lse, 0.0), ze


def backward(x, w, dloss, q, has, T=1.0):
    """dx, dw of sum dloss loss, and dz [N,V]; q as target_weights or teacher_weights return it."""
    rows = torch.nonzero(has).view(-1)
    xr, wd = x[rows].double(), w.double()
    p = torch.softmax(xr @ wd.t() / T, 1)
    dz = (p - q[rows]) * (dloss[rows].double() / T)[:, None]
    dx = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    dx[rows] = dz @ wd
    full = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device=x.device)
    full[rows] = dz
    return dx, dz.t() @ xr, full
