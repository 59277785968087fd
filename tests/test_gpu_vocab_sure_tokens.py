"""Cross entropy of tokens whose probability is 1 or next to it: lse and the target's logit are the same number but for rounding.  The
loss is 0 at least and accurate to its own size, and the gradient at the target points the other way or nowhere.

Tolerances as in test_gpu_vocab_loss.py, whose check() is applied too."""
import pytest
import torch

from test_gpu_vocab_loss import DEV, HALF, U, call, check, make

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


def _exact(x, w, target):
    """The loss as log(1 + sum over the others of exp(z - z[target])), in 64 bits, and what a logit is made of at most."""
    x, w = x.double(), w.double()
    z = x @ w.t()
    at = target.long()[:, None]
    d = torch.logsumexp(z.scatter(1, at, -torch.inf), 1) - torch.gather(z, 1, at)[:, 0]
    return torch.clamp(d, min=0) + torch.log1p(torch.exp(-d.abs())), d, (x.abs() @ w.abs().t()).max(1).values


def _relative(M, d, S_abs):
    """With d the log-sum of the other entries less the target's logit, loss = log(1 + e^d): an error of d is one of at most
    as much relative to the loss (its derivative is 1 - e^-loss).  d: two logits and the sum, as in test_gpu_vocab_loss.py, and
    8 u of what it is made of."""
    return 2 * 2 * (M + 2) * U * S_abs + 2 ** 10 * U + 8 * U * (d.abs() + 1)


# tokens from uncertain to all but certain, in each form of the products and of the passes over rows
NEARLY = [(1, 64, 2, "bf16"), (5, 1024, 900, "bf16"), (5, 512, 900, "f32"), (60, 136, 515, "bf16"), (200, 264, 8000, "bf16"), (300, 260, 1001, "f32"),
          (1500, 72, 3001, "f32"), (1000, 520, 1500, "bf16"), (2100, 448, 33333, "bf16"), (1024, 1024, 32000, "bf16")]


@pytest.mark.parametrize("S,M,V,dtype", NEARLY)
def test_small_losses_to_their_own_size(S, M, V, dtype):
    d = make(1, S, M, V, dtype, 0.1 if S > 5 else 0.0)
    has = d["target"] >= 0
    sure = torch.linspace(12.0, 1.0, S, device=DEV)[:, None]
    d["x"] = (sure * d["w"][d["target"].clamp(min=0).long()].float() + 0.1 * d["x"].float()).to(d["x"].dtype)
    r = call(1, S, M, V, dtype, d, backward=False)
    want, off, S_abs = _exact(d["x"][has], d["w"], d["target"][has])
    assert want.min() < 1e-4
    ratio = ((r["loss"][has].double() - want).abs() / (want * _relative(M, off, S_abs) + 2.0 ** -126)).max().item()
    assert ratio <= 1
    assert (r["loss"][~has] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 3.0, 6.0, 12.0])
def test_gradient_of_a_sure_target(dtype, scale):
    """dw of a single token's target is dz x: to the size of dz, however small.  dz is rounded to the element type, and the product."""
    M, V = 256, 700
    d = make(1, 1, M, V, dtype)
    d["x"] = (scale * d["w"][d["target"].long()].float()).to(d["x"].dtype)
    r = call(1, 1, M, V, dtype, d)
    loss, off, S_abs = _exact(d["x"], d["w"], d["target"])
    want = d["dloss"].double() * torch.expm1(-loss) * d["x"][0].double()
    t = want.abs() * (_relative(M, off, S_abs) + 16 * U + 3 * HALF[dtype]) + 2.0 ** -126
    ratio = ((r["dw"][d["target"][0].long()].double() - want).abs() / t).max().item()
    assert ratio <= 1


@pytest.mark.parametrize("S,M,V,dtype", [(257, 64, 257, "bf16"), (60, 72, 60, "bf16"), (1030, 136, 515, "bf16"), (700, 520, 700, "bf16"), (255, 36, 255, "f32"),
                                         (1030, 260, 515, "f32"), (700, 516, 700, "f32"), (2304, 1024, 9000, "bf16"), (2100, 448, 33333, "bf16")])
def test_targets_in_every_column(S, M, V, dtype):
    """Each column of a tile is some row's target, the last one of the vocabulary among them, and rows of a tile share one."""
    d = make(1, S, M, V, dtype)
    d["target"] = (V - 1 - torch.arange(S, device=DEV) * (1 if V <= S else 17) % V).int()
    d["target"][S // 2:S // 2 + 9] = V // 2
    check(1, S, M, V, dtype, d, call(1, S, M, V, dtype, d))
