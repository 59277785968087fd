"""The losses over a vocabulary and their gradients against the 64-bit oracle.

Tolerances, from the number of roundings.  u = 2^-24.  A logit is a sum of M products: each of the M additions (and for fp32 the
terms that a product leaves out) is off by at most u of a partial sum, so |dz_logit| <= 2 (M + 2) u S with S = max_v sum_m |x w|.
lse and loss: that, two roundings per slot, lane and step of the sum (fewer than 2^9 of 2u), and 8 u of what is subtracted.
A gradient dz is p times the relative error that the errors of z and lse make (each at most the above), rounded once to the
element type (half a step: 2^-8 bf16, 2^-24 fp32); dx and dw sum those errors, add (terms) u of the sum of magnitudes, and are
rounded once.  Both types' smallest normal number is 2^-126, and the power of two gives 0 below it: a p under 2^-126 is off by up
to 2^-126 (times the upstream gradient), a dz under 2^-126 too.  (A logit 87 under its lse gets there: test_far_logits, whose x of
a few hundred make 1e-36 of it.)
"""
import pytest
import torch

import paper_2006_16668_amd as moe
from oracle import vocab_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": U}


def make(G, S, M, V, dtype, empty=0.0, K=0, seed=0, sure=2.0):
    g = torch.Generator(device=DEV).manual_seed(1000003 * seed + G * S * M + V + K)
    N = G * S
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    w = (rand(V, M) * (2.0 / M ** 0.5)).to(DT[dtype])
    t = torch.randint(0, V, (N,), generator=g, device=DEV)
    x = (rand(N, M) + sure * torch.rand(N, 1, generator=g, device=DEV) * w[t].float()).to(DT[dtype])
    out = {"x": x, "w": w, "dloss": torch.rand(N, generator=g, device=DEV) / N}
    gone = torch.rand(N, generator=g, device=DEV) < empty
    if K:
        idx = torch.randint(0, V, (N, K), generator=g, device=DEV)
        idx[:, 0] = t
        idx = torch.where((torch.rand(N, K, generator=g, device=DEV) < 0.1) | gone[:, None], -1, idx)
        out.update(idx=idx.int(), logit=2 * rand(N, K))
    else:
        out["target"] = torch.where(gone, -1, t).int()
    return out


def call(G, S, M, V, dtype, d, K=0, T=1.0, piece=0, backward=True, ws_fill=0xff):
    """Both passes through the public entry points; everything written starts as NaN."""
    sh, dims = moe.MoEShape(G, S, M, M, 2, 1, dtype), moe.VocabDims(V, K=K, temperature=T, piece=piece)
    f = lambda *s: torch.full(s, float("nan"), device=DEV)
    ws = torch.full((moe.moe_vocab_workspace_bytes(sh, dims),), ws_fill, dtype=torch.uint8, device=DEV)
    r = {"loss": f(G, S), "lse": f(G, S)}
    x = d["x"].view(G, S, M)
    if K:
        r["entry_logit"] = f(G, S, K)
        idx, logit = d["idx"].view(G, S, K), d["logit"].view(G, S, K)
        moe.moe_vocab_distill(sh, dims, x, d["w"], idx, logit, r["loss"], r["lse"], r["entry_logit"], ws)
    else:
        target = d["target"].view(G, S)
        moe.moe_vocab_loss(sh, dims, x, d["w"], target, r["loss"], r["lse"], ws)
    if backward:
        dloss = d["dloss"].view(G, S)
        r["dx"], r["dw"] = torch.full_like(x, float("nan")), torch.full_like(d["w"], float("nan"))
        bws = torch.full((moe.moe_vocab_backward_workspace_bytes(sh, dims),), ws_fill, dtype=torch.uint8, device=DEV)
        if K:
            moe.moe_vocab_distill_backward(sh, dims, x, d["w"], idx, logit, r["entry_logit"], r["lse"], dloss, r["dx"], r["dw"], bws)
        else:
            moe.moe_vocab_loss_backward(sh, dims, x, d["w"], target, r["loss"], r["lse"], dloss, r["dx"], r["dw"], bws)
    torch.cuda.synchronize()
    return {k: v.reshape(-1, *v.shape[2:]) if k != "dw" else v for k, v in r.items()}


def check(G, S, M, V, dtype, d, r, K=0, T=1.0):
    N = G * S
    x, w = d["x"], d["w"]
    if K:
        q, has, _, there = orc.teacher_weights(N, V, d["idx"], d["logit"], T, DEV)
        loss, lse, ze = orc.distill(x, w, d["idx"], d["logit"], T)
    else:
        q, has = orc.target_weights(N, V, d["target"], DEV)
        loss, lse = orc.cross_entropy(x, w, d["target"])
    S_abs = (x.double().abs() @ w.double().abs().t()).max(1).values
    dz = 2 * (M + 2) * U * S_abs / T
    tol = dz + 2 ** 10 * U + 8 * U * (lse.abs() + S_abs / T)
    for k, want in (("lse", lse), ("loss", loss)):
        err = (r[k].double() - want).abs()
        bound = tol if k == "lse" else 2 * tol                   # (lse and a logit)
        assert (err <= bound)[has].all(), (k, (err / bound)[has].max().item())
        assert (r[k][~has] == 0).all(), k
    if K:
        err = (r["entry_logit"].double() - ze).abs()
        assert (err <= (dz * T)[:, None] + U * ze.abs()).all()
        assert (r["entry_logit"][~there] == 0).all()
    if "dx" not in r:
        return
    dx, dw, grad = orc.backward(x, w, d["dloss"], q, has, T)
    up = (d["dloss"].double() / T * has)[:, None]
    p = grad / torch.where(up > 0, up, 1.0) + q * has[:, None]
    e = up * (p + q) * 2 * tol[:, None] + 16 * U * (up * (p + q)) + HALF[dtype] * grad.abs()
    e += 2.0 ** -126 * (1 + up) * has[:, None]
    wa, xa = w.double().abs(), torch.where(has[:, None], x.double(), 0.0).abs()
    mag = grad.abs() + e
    tx = e @ wa + (V + 64) * 2 * U * (mag @ wa) + HALF[dtype] * dx.abs() + 2.0 ** -126
    tw = e.t() @ xa + (N + 64) * 2 * U * (mag.t() @ xa) + HALF[dtype] * dw.abs() + 2.0 ** -126
    for k, want, t in (("dx", dx, tx), ("dw", dw, tw)):
        got = r[k].double()
        assert torch.isfinite(got).all(), k
        ratio = ((got - want).abs() / (t + HALF[dtype] * t)).max().item()
        assert ratio <= 1.0, (k, ratio)
    assert (r["dx"][~has] == 0).all()


# G, S, M, V, dtype, share without a target, piece
CE = [(1, 64, 128, 900, "bf16", 0.5, 0), (1, 33, 72, 515, "f32", 0.5, 0), (5, 13, 256, 2100, "bf16", 0.2, 512), (2, 31, 64, 70, "bf16", 0.9, 0),
      (1, 1, 8, 1, "bf16", 0, 0), (1, 1, 4, 1, "f32", 0, 0), (1, 1, 64, 2, "bf16", 0, 0), (1, 3, 40, 17, "bf16", 0, 0),
      (1, 3, 36, 17, "f32", 0, 0), (2, 65, 72, 257, "bf16", 0.3, 0), (2, 65, 68, 255, "f32", 0.3, 0), (1, 300, 264, 1000, "bf16", 0, 256),
      (3, 100, 520, 515, "bf16", 0.7, 256), (3, 100, 260, 515, "f32", 0.7, 256), (1, 1, 1024, 4001, "bf16", 0, 0),
      (1, 17, 512, 8193, "f32", 0.1, 0), (1, 1025, 128, 1031, "bf16", 0.5, 512), (1, 2049, 32, 300, "bf16", 0.05, 0),
      (4, 1000, 200, 3001, "bf16", 0.1, 0), (1, 5000, 256, 12000, "bf16", 0.1, 0), (1, 3000, 1000, 2500, "f32", 0.1, 1024),
      # products on 256 x 256 tiles (test_vocab_rules.py: which): ragged in every dimension, several pieces, the last of few entries,
      # most rows without a target
      (1, 2100, 448, 33333, "bf16", 0.1, 0), (3, 1021, 776, 20257, "bf16", 0.6, 0), (1, 6000, 192, 9999, "bf16", 0.3, 0),
      (1, 3000, 1000, 9001, "bf16", 0, 4096), (2, 1250, 1344, 7003, "bf16", 0.02, 0), (1, 32, 4096, 16000, "bf16", 0, 0),
      (1, 1024, 1024, 32000, "bf16", 0.97, 0), (1, 2048, 1024, 32000, "bf16", 0.05, 0),
      (1, 9001, 72, 26001, "bf16", 0, 8192),
      # dw summed over ranges of the rows: ragged ones, hardly any row, one piece of the vocabulary after the other
      (1, 5003, 216, 461, "bf16", 0.2, 0), (3, 3001, 152, 211, "bf16", 0.995, 0), (1, 12001, 72, 1030, "bf16", 0.4, 512),
      (1, 3001, 68, 701, "f32", 0.3, 0), (7, 701, 36, 333, "f32", 0.995, 0), (1, 6001, 100, 515, "f32", 0, 256)]


@pytest.mark.parametrize("G,S,M,V,dtype,empty,piece", CE)
def test_cross_entropy(G, S, M, V, dtype, empty, piece):
    d = make(G, S, M, V, dtype, empty)
    check(G, S, M, V, dtype, d, call(G, S, M, V, dtype, d, piece=piece))


# G, S, M, V, K, T, dtype, share without, piece
KD = [(1, 64, 72, 300, 20, 2.0, "bf16", 0.5, 0), (5, 8, 132, 700, 3, 1.5, "f32", 0.4, 0), (1, 63, 256, 2048, 256, 1.0, "bf16", 0.1, 0),
      (1, 1, 8, 1, 1, 1.0, "bf16", 0, 0), (1, 5, 40, 3, 9, 0.5, "bf16", 0, 0), (1, 5, 36, 33, 3, 2.0, "f32", 0.2, 0),
      (2, 65, 72, 257, 16, 2.0, "bf16", 0.3, 0), (1, 200, 136, 1500, 65, 3.0, "bf16", 0.1, 256), (1, 77, 68, 700, 256, 1.0, "f32", 0.1, 256),
      (1, 1, 1024, 4001, 31, 4.0, "bf16", 0, 0), (2, 1100, 256, 2999, 32, 2.0, "bf16", 0.1, 0),
      # the product leaves the logits at the entries (test_vocab_rules.py)
      (1, 2500, 1024, 16001, 32, 2.0, "bf16", 0.2, 0), (3, 700, 520, 31011, 256, 1.0, "bf16", 0.1, 8192), (1, 4096, 256, 33000, 100, 3.0, "bf16", 0, 0),
      # a product that is on tiles for that reason
      (1, 6011, 520, 1111, 40, 2.0, "bf16", 0.4, 0)]


@pytest.mark.parametrize("G,S,M,V,K,T,dtype,empty,piece", KD)
def test_distillation(G, S, M, V, K, T, dtype, empty, piece):
    d = make(G, S, M, V, dtype, empty, K)
    check(G, S, M, V, dtype, d, call(G, S, M, V, dtype, d, K, T, piece), K, T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 5])
def test_no_token_and_one_token_with_a_target(dtype, K):
    for G, S, M, V, keep in [(2, 700, 64, 777, k) for k in ([], [1399], [0], [63, 64, 1023, 1024])] + \
            [(1, 9000, 64, 300, k) for k in ([], [8999])] + \
            [(1, 64, 72, 777, k) for k in ([], [63], [0], [5, 6])]:
        d = make(G, S, M, V, dtype, K=K)
        gone = torch.ones(G * S, dtype=torch.bool, device=DEV)
        gone[keep] = False
        # what tokens without a target hold is not used
        d["x"][gone] = float("nan")
        d["dloss"][gone] = float("inf")
        if K:
            d["idx"][gone] = V + 7
        else:
            d["target"][gone] = torch.randint(V, 2 ** 31 - 1, (int(gone.sum()),), device=DEV, dtype=torch.int32)
        r = call(G, S, M, V, dtype, d, K)
        clean = dict(d, x=torch.where(gone[:, None], 0, d["x"]), dloss=torch.where(gone, 0, d["dloss"]))
        check(G, S, M, V, dtype, clean, r, K)
        if not keep:
            assert (r["dw"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_teacher_lists_with_gaps(dtype):
    """-inf and lowest logits, one index many times, entries outside the vocabulary."""
    G, S, M, V, K = 1, 8, 64, 100, 6
    d = make(G, S, M, V, dtype, K=K)
    low = torch.finfo(torch.float32).min
    d["idx"].clamp_(min=0)
    d["logit"][0] = low                                          # all the lowest: alike
    d["logit"][1] = -torch.inf                                   # none there
    d["logit"][2, 1:] = low                                      # one that counts
    d["logit"][3, ::2] = -torch.inf
    d["idx"][4] = 42
    d["idx"][5] = torch.tensor([7, 7, 8, -1, 8, V], dtype=torch.int32, device=DEV)
    d["idx"][6] = torch.iinfo(torch.int32).min
    d["idx"][7], d["logit"][7] = V - 1, low
    for T in (0.25, 1.0, 8.0):
        check(G, S, M, V, dtype, d, call(G, S, M, V, dtype, d, K, T), K, T)


def test_entries_crowded_into_few_tiles():
    """More entries in a 256 x 256 tile of the logits than a wavefront has lanes, many of them the same."""
    G, S, M, V, K = 1, 2100, 1032, 17000, 64
    d = make(G, S, M, V, "bf16", 0.1, K)
    there = d["idx"] >= 0
    d["idx"] = torch.where(there & (torch.arange(K, device=DEV) > 0), 16640 + d["idx"] % 360, d["idx"]).int()
    check(G, S, M, V, "bf16", d, call(G, S, M, V, "bf16", d, K, 2.0), K, 2.0)


def test_far_logits():
    """Differences of hundreds between logits, a certain token, and one whose target is out of reach: no overflow, no NaN."""
    G, S, M, V = 1, 6, 64, 1000
    for dtype in ("bf16", "f32"):
        d = make(G, S, M, V, dtype)
        d["x"] *= 64
        d["target"][0] = (d["x"][0].double() @ d["w"].double().t()).argmax().int()
        d["target"][1] = (d["x"][1].double() @ d["w"].double().t()).argmin().int()
        d["x"][2] = 0
        check(G, S, M, V, dtype, d, call(G, S, M, V, dtype, d))


def test_numbers_that_are_not_finite_stay_in_their_rows():
    """A row of x with NaN or an infinity, which has a target, spoils its own loss and dx and all of dw, and no other row's."""
    G, S, M, V = 1, 200, 64, 500
    for dtype in ("bf16", "f32"):
        d = make(G, S, M, V, dtype)
        clean = call(G, S, M, V, dtype, d, backward=False)
        d["x"][70, 3], d["x"][130, 5] = float("nan"), float("inf")
        r = call(G, S, M, V, dtype, d)
        rest = torch.ones(S, dtype=torch.bool, device=DEV)
        rest[[70, 130]] = False
        if dtype == "bf16":
            assert torch.equal(r["loss"][rest], clean["loss"][rest])
        # (fp32: tiles with such a result are multiplied again, in the products that the instruction for fp32 forms: both sums
        # of the other rows are within the bound of one)
        S_abs = (d["x"][rest].double().abs() @ d["w"].double().abs().t()).max(1).values
        tol = 2 * (M + 2) * U * S_abs + 2 ** 10 * U + 8 * U * (clean["lse"][rest].abs() + S_abs)
        assert ((r["loss"][rest] - clean["loss"][rest]).abs() <= 4 * tol).all() and torch.isfinite(r["dx"][rest]).all()
        assert not torch.isfinite(r["loss"][~rest]).any() and not torch.isfinite(r["dx"][~rest].float()).all(1).any()


@pytest.mark.parametrize("K", [0, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_again(dtype, K):
    """No result depends on the order of blocks, nor on what the workspace held; pieces change no loss."""
    G, S, M, V = 1, 900, 136, 2500
    d = make(G, S, M, V, dtype, 0.2, K)
    a, b = (call(G, S, M, V, dtype, d, K, 2.0, ws_fill=f) for f in (0x00, 0xff))
    for k in a:
        assert torch.equal(a[k], b[k]), k
