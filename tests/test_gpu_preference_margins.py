"""Preference losses of long sequences whose ratios are large and nearly equal, from the token losses to the gradient, against 64 bits.

u = 2^-24.  The loss comes from sums in 64 bits: one rounding, u, and what remains of those sums' own (n 2^-53 of their terms' magnitudes, times the slope).  The
gradient is formed at the ratios as they are stored: h off by u (|r0| + |r1|), d loss / d h by beta^2 / 4 (the largest derivative of beta sigmoid(beta h); the
terms of a smoothed loss share it) or 2 of that, then one rounding, u."""
import pytest
import torch

import paper_2006_16668_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("kind,beta,e", [("logistic", 0.1, 0.0), ("logistic", 1.0, 0.2), ("squared", 0.5, 0.0)])
@pytest.mark.parametrize("size", [1.0, 100.0, 1e4, 1e6])
def test_margin_of_large_ratios(size, kind, beta, e):
    g = torch.Generator(device=DEV).manual_seed(int(size))
    P, S, V = 3, 2001, 100
    nll = 2 * torch.rand(2 * P, S, generator=g, device=DEV) + 0.1
    ref = nll + size / S * (1 + 0.1 * torch.randn(2 * P, S, generator=g, device=DEV))
    by = (ref.double() - nll.double()).sum(1)
    ref[1::2, 0] += (by[0::2] - by[1::2] - torch.tensor([1.0, -0.6, 0.2], device=DEV, dtype=torch.float64)).float()      # margins of about these
    target = torch.zeros(2 * P, S, dtype=torch.int32, device=DEV)
    start = torch.arange(0, 2 * P * S + 1, S, dtype=torch.int32, device=DEV)
    dloss = torch.rand(P, generator=g, device=DEV) + 0.5
    sh, dims = moe.MoEShape(2 * P, S, 8, 8, 2, 1, "f32"), moe.PreferenceDims(P, V, beta, e, kind)
    loss, ratio, dnll = (torch.full(s, float("nan"), device=DEV) for s in ((P,), (2 * P,), (2 * P, S)))
    moe.moe_preference_loss(sh, dims, nll, ref, target, start, loss, ratio)
    moe.moe_preference_loss_backward(sh, dims, target, start, ratio, dloss, dnll)
    terms = ref.double() - nll.double()
    r = terms.sum(1)
    h = r[0::2] - r[1::2]
    assert (h.abs() < 1.2).all() and (size < 100 or (r.abs() >= 0.5 * size).all())          # (what the inputs are to be: the margin is of a ratio of 1 all of it)
    sig, sp = torch.sigmoid, torch.nn.functional.softplus
    if kind == "logistic":
        want = (1 - e) * sp(-beta * h) + e * sp(beta * h)
        slope, curve = beta * (sig(beta * h) - (1 - e)), beta * beta / 4
    else:
        want, slope, curve = (h - 0.5 / beta) ** 2, 2 * (h - 0.5 / beta), 2.0
    e_sum = S * 2.0 ** -53 * terms.abs().sum(1).view(P, 2).sum(1) * 2
    assert ((loss.double() - want).abs() <= 1.01 * U * want + slope.abs() * e_sum + curve * e_sum ** 2).all()
    e_h = U * r.abs().view(P, 2).sum(1) + e_sum
    err = (curve * e_h + 1.01 * U * (slope.abs() + curve * e_h)) * dloss
    for s in range(2):
        got = dnll[s::2].double()
        assert (got == got[:, :1]).all()                        # one value for all tokens of a sequence
        assert ((got[:, 0] - (1 if s else -1) * slope * dloss).abs() <= err).all()
