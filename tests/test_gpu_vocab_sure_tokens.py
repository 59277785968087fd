"""Cross entropy of tokens whose probability is 1 or next to it: lse and the target's logit are the same number but for rounding, summed
in different orders.  The loss is 0 at least, and the gradient at the target points the other way or nowhere.

Tolerances as in test_gpu_vocab_loss.py, whose check() is applied too."""
import pytest
import torch

from test_gpu_vocab_loss import DEV, call, check, make

pytestmark = pytest.mark.gpu

# one entry; each form of the products and of the passes over rows: few tokens, up to 1024, more, 256 x 256 tiles
SIZES = [(1, 33, 1024, 1), (1, 700, 1000, 1), (1, 1500, 520, 1), (1, 60, 1024, 700), (1, 900, 256, 515), (1, 2100, 448, 33333)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,S,M,V", SIZES)
def test_no_loss_below_zero(G, S, M, V, dtype):
    if dtype == "f32" and V > 20000:
        S, V = 300, 9999
    d = make(G, S, M, V, dtype, 0.1)
    sure = d["target"] >= 0
    if V > 1:
        d["x"] = torch.where(sure[:, None], 12.0 * d["w"][d["target"].clamp(min=0).long()].float(), d["x"].float()).to(d["x"].dtype)
    r = call(G, S, M, V, dtype, d)
    check(G, S, M, V, dtype, d, r)
    assert (r["loss"] >= 0).all(), r["loss"].min().item()
    assert (r["loss"][sure] < 1e-3).all()
    if V == 1:                                                   # dx = dz w: along w or nothing
        assert ((r["dx"].double() @ d["w"][0].double()) <= 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_stays(dtype):
    d = make(1, 70, 64, 1, dtype)
    d["x"][5, 3] = float("nan")
    r = call(1, 70, 64, 1, dtype, d, backward=False)
    assert torch.isnan(r["loss"][5]) and (r["loss"][torch.arange(70, device=DEV) != 5] >= 0).all()
