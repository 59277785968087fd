"""The losses of preference and policy read G and S of a configuration and nothing else: what a caller without experts leaves there is no reason to refuse."""
import pytest
import torch

import paper_2006_16668_amd as moe
from paper_2006_16668_amd.binding import _PolicyDims, _PreferenceDims
from test_decoder_limits import EINVAL, EUNSUPPORTED, VP, call
from test_vocab_rules import _C

CALLS = [("moe_preference_loss", _PreferenceDims(2, 9, 0, 0.1, 0.0), 6), ("moe_preference_loss_backward", _PreferenceDims(2, 9, 0, 0.1, 0.0), 5),
         ("moe_policy_loss", _PolicyDims(9, 1, 0.2, 0.2, 0.1), 7), ("moe_policy_loss_backward", _PolicyDims(9, 1, 0.2, 0.2, 0.1), 7)]


@pytest.mark.parametrize("name,dims,n", CALLS)
def test_other_fields_do_not_count(name, dims, n):
    """A missing address is found after the configuration."""
    for cfg in (_C(2, 8, 1, 8, 2, 1, 1), _C(2, 8, 0, 0, 0, 0, 0), _C(2, 8, 64, 64, 1, 1, 9), _C(2, 8, 7, -3, 1 << 30, 1 << 30, -1)):
        assert call(name, cfg, dims, [VP(0)] * n + [None]) == EINVAL
    for cfg, status in ((_C(0, 8, 8, 8, 2, 1, 0), EINVAL), (_C(2, 0, 8, 8, 2, 1, 0), EINVAL), (_C(-2, -8, 8, 8, 2, 1, 0), EINVAL),
                        (_C(1 << 15, 1 << 15, 8, 8, 2, 1, 0), EUNSUPPORTED), (_C((1 << 15) - 1, 1 << 15, 1, 0, 0, 0, 0), EINVAL)):
        assert call(name, cfg, dims, [VP(0)] * n + [None]) == status


@pytest.mark.gpu
def test_results_are_those_of_a_whole_configuration():
    g = torch.Generator(device="cuda:0").manual_seed(0)
    G, S, P = 4, 37, 2
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda:0") + 0.1
    nll, ref, old, adv, up, pup = rand(G, S), rand(G, S), rand(G, S), rand(G) - 0.6, rand(G, S), rand(P)
    target = torch.randint(-1, 9, (G, S), generator=g, device="cuda:0", dtype=torch.int32)
    start = torch.arange(0, G * S + 1, S, dtype=torch.int32, device="cuda:0")
    results = []
    for sh in (moe.MoEShape(G, S, 8, 8, 2, 1, "f32"), moe.MoEShape(G, S, 1, 0, 0, 0)):
        pd, qd = moe.PreferenceDims(P, 9, 0.3), moe.PolicyDims(9, 0.2, 0.2, 0.1)
        loss, ratio, dnll, ploss, kl, pdnll = (torch.full(s, float("nan"), device="cuda:0") for s in ((P,), (2 * P,), (G, S), (G, S), (G, S), (G, S)))
        moe.moe_preference_loss(sh, pd, nll, ref, target, start, loss, ratio)
        moe.moe_preference_loss_backward(sh, pd, target, start, ratio, pup, dnll)
        moe.moe_policy_loss(sh, qd, nll, old, ref, adv, target, ploss, kl)
        moe.moe_policy_loss_backward(sh, qd, nll, old, ref, adv, target, up, pdnll)
        results.append((loss, ratio, dnll, ploss, kl, pdnll))
    for a, b in zip(*results):
        assert torch.isfinite(a).all() and torch.equal(a, b)
