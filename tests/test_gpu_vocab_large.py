"""The losses over a vocabulary where offsets pass 32 bits: tokens behind 4 GiB of x, rows of the logits' gradient 16 MB apart, and
the largest vocabulary.

Tolerances as in test_gpu_vocab_loss.py (u = 2^-24, h the half step of the element type)."""
import pytest
import torch

import paper_2006_16668_amd as moe
from test_gpu_vocab_loss import DEV, DT, HALF, U, call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,M", [("bf16", (1 << 20) + 77, 2176), ("f32", (1 << 20) + 77, 1088)])
def test_tokens_behind_4_gib(dtype, N, M):
    """Most tokens have a target, a few at either end a gradient: theirs are checked as a call of their own would be, and all that
    reaches dw is from them."""
    V, keep = 333, 24
    g = torch.Generator(device=DEV).manual_seed(N)
    w = (torch.randn(V, M, generator=g, device=DEV) * (2.0 / M ** 0.5)).to(DT[dtype])
    x = torch.empty(N, M, dtype=DT[dtype], device=DEV)
    for r in range(0, N, 1 << 17):
        x[r:r + (1 << 17)] = torch.randn(min(1 << 17, N - r), M, generator=g, device=DEV).to(DT[dtype])
    assert x.numel() * x.element_size() > 1 << 32
    target = torch.randint(0, V, (N,), generator=g, device=DEV).int()
    target[keep:N - keep][torch.rand(N - 2 * keep, generator=g, device=DEV) < 0.1] = -1
    dloss = torch.zeros(N, device=DEV)
    few = torch.cat([torch.arange(keep, device=DEV), torch.arange(N - keep, N, device=DEV)])
    dloss[few] = 0.5 + torch.rand(2 * keep, generator=g, device=DEV)
    d = {"x": x, "w": w, "target": target, "dloss": dloss}
    r = call(1, N, M, V, dtype, d)
    assert torch.equal(r["loss"] > 0, target >= 0)               # (a target's probability is far from 1 here)
    part = {k: v[few] if k != "w" else v for k, v in d.items()}
    check(1, 2 * keep, M, V, dtype, part, {k: v[few] if k != "dw" else v for k, v in r.items()})
    dx = r["dx"]
    dx[few] = 0
    assert all((dx[i:i + (1 << 17)] == 0).all() for i in range(0, N, 1 << 17))       # (and nowhere NaN)


def test_largest_vocabulary_in_one_piece():
    """2^23 entries.  dz in one piece, in rows of 16 MB, and in several: the same dz, so dw bit for bit.  dx is a sum of the pieces'
    sums: each of at most 2^23 / 16 steps, off by u of a partial sum each, that is by 2^-5 of sum |dz| |w| at worst, where sum |dz|
    is at most 2 dloss; it is summed in 64 ranges (few tiles, a long sum), so 2^-11 of 2 dloss max |w| and as much again for all other
    additions, twice for the two; and both are rounded once."""
    N, M, V = 256, 72, 1 << 23
    g = torch.Generator(device=DEV).manual_seed(5)
    w = torch.empty(V, M, dtype=torch.bfloat16, device=DEV)
    for r in range(0, V, 1 << 20):
        w[r:r + (1 << 20)] = torch.randn(1 << 20, M, generator=g, device=DEV).to(torch.bfloat16)
    x = (torch.randn(N, M, generator=g, device=DEV) * 0.5).to(torch.bfloat16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV).int()
    target[0], target[-1] = V - 1, V - 1                         # one entry twice, the last
    d = {"x": x, "w": w, "target": target, "dloss": 0.5 + torch.rand(N, generator=g, device=DEV)}
    one, many = (call(1, N, M, V, "bf16", d, piece=p) for p in (V, 1 << 20))
    for k in ("loss", "lse", "dw"):
        assert torch.equal(one[k], many[k]), k
    a, b = one["dx"].double(), many["dx"].double()
    most = w.abs().max().double() * 2 * d["dloss"].double()[:, None]
    assert ((a - b).abs() <= 2 * 2.0 ** -10 * most + HALF["bf16"] * (a.abs() + b.abs())).all()
    # the loss of some rows, in 64 bits
    rows = [0, 1, 128, 255]
    z = torch.cat([x[rows].double() @ w[r:r + (1 << 20)].double().t() for r in range(0, V, 1 << 20)], 1)
    lse = torch.logsumexp(z, 1)
    S_abs = max((x[rows].double().abs() @ w[r:r + (1 << 20)].double().abs().t()).max() for r in range(0, V, 1 << 20))
    tol = 2 * (M + 2) * U * S_abs + 2 ** 10 * U + 8 * U * (lse.abs() + S_abs)
    assert ((one["lse"][rows].double() - lse).abs() <= tol).all()
    assert ((one["loss"][rows].double() - (lse - z[torch.arange(4), target[rows].long()])).abs() <= 2 * tol).all()
    # dw of the rows around the border of 4 GiB of dz, and the last: sum over tokens of dz x, in 64 bits from the lse above
    x64, up = x.double(), d["dloss"].double()[:, None]
    for v in ((1 << 23) - 512, (1 << 22) - 256, 0):
        p = torch.exp(x64 @ w[v:v + 512].double().t() - one["lse"].double()[:, None])
        hit = target.long()[:, None] == torch.arange(v, v + 512, device=DEV)
        dz = up * (p - hit.double())
        want = dz.t() @ x64
        e = dz.abs() * HALF["bf16"] + up * (p + hit) * 4 * tol.max() + 2.0 ** -126 * (1 + up)
        t = e.t() @ x64.abs() + (N + 64) * 2 * U * ((dz.abs() + e).t() @ x64.abs()) + HALF["bf16"] * want.abs() + 2.0 ** -126
        assert ((one["dw"][v:v + 512].double() - want).abs() <= t * (1 + HALF["bf16"])).all(), v
