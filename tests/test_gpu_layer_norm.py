"""moe_add_layer_norm for rows of any width and its derivative against the formulas in 64 bits.

Tolerances.  u = 2^-24, h the half step of the element type (bf16 2^-8, fp32 u).  A row's mean and its sums of M terms are off by at
most M u of the mean magnitude of the terms; xhat = (s - mean) rstd then by e = 4 M u (1 + |xhat|) at most (mean, variance and
root, each below M u relative to the row's spread; rows here have a mean of at most ten times their spread).  n is rounded once;
ds sums three terms with those errors and is rounded once; dgamma and dbeta add up rows terms.
"""
import pytest
import torch

import paper_2006_16668_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": U}


def make(G, S, M, dtype, residual, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + G * S * 31 + M)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x = (rand(G, S, M) * (0.3 + torch.rand(G, S, 1, generator=g, device=DEV)) + rand(G, S, 1)).to(DT[dtype])
    return {"x": x, "delta": rand(G, S, M).to(DT[dtype]) if residual else None, "gamma": 1 + 0.3 * rand(M), "beta": rand(M),
            "dn": rand(G, S, M).to(DT[dtype]), "dres": rand(G, S, M).to(DT[dtype]) if residual else None}


def xhat(s):
    s = s.double()
    c = s - s.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6)
    return c * rstd, rstd


# wavefronts (with many rows up to 3 or 5 KB, else 8 KB backward); blocks, one to four vectors a thread backward; any
WIDTHS = [("bf16", M) for M in (8, 520, 4096, 4104, 8192, 8200, 12288, 12296, 16384, 16392, 40000)] + \
         [("bf16", M) for M in (1024, 1536, 1544, 2400, 2800)] + \
         [("f32", M) for M in (4, 260, 520, 1024, 1196, 1284, 1500, 2048, 2052, 4100, 8192, 8196, 20004)]


# (many rows: once per form)
CASES = [(dtype, M, G, S, residual) for dtype, M in WIDTHS for G, S in ((1, 1), (3, 7), (1, 1111)) for residual in (False, True)
         if S < 1000 or not (M > 17000 or residual and M < 4000)]


@pytest.mark.parametrize("dtype,M,G,S,residual", CASES)
def test_forward_and_backward(dtype, M, G, S, residual):
    d = make(G, S, M, dtype, residual)
    sh = moe.MoEShape(G, S, M, M, 2, 1, dtype)
    nan = lambda t: torch.full_like(t, float("nan"))
    s_out, n_out = (nan(d["x"]) if residual else None), nan(d["x"])
    moe.moe_add_layer_norm(sh, d["x"], d["delta"], d["gamma"], d["beta"], s_out, n_out)
    s = d["x"]
    if residual:
        want = d["x"].double() + d["delta"].double()
        assert ((s_out.double() - want).abs() <= (HALF[dtype] + U) * want.abs()).all()
        s = s_out
    xh, rstd = xhat(s)
    e = 4 * M * U * (1 + xh.abs())
    want = d["gamma"].double() * xh + d["beta"].double()
    tol = d["gamma"].double().abs() * e + HALF[dtype] * want.abs() + 4 * U * (want.abs() + d["beta"].double().abs())
    assert ((n_out.double() - want).abs() <= tol).all()

    ds, dgamma, dbeta = nan(s), nan(d["gamma"]), nan(d["beta"])
    ws = torch.full((moe.moe_layer_norm_backward_workspace_bytes(sh),), 0xff, dtype=torch.uint8, device=DEV)
    moe.moe_add_layer_norm_backward(sh, s, d["dn"], d["gamma"], d["dres"], ds, dgamma, dbeta, ws)
    dn = d["dn"].double()
    g = dn * d["gamma"].double()
    want = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    size = rstd * (g.abs() + g.abs().mean(-1, keepdim=True) + xh.abs() * (g * xh).abs().mean(-1, keepdim=True))
    if residual:
        want = want + d["dres"].double()
    # each of the three terms is off by e of its size, relative to a spread of 1
    tol = 8 * M * U * size * (1 + xh.abs()) + HALF[dtype] * want.abs() + 4 * U * want.abs()
    assert ((ds.double() - want).abs() <= tol).all()
    rows = G * S
    for got, terms, err in ((dgamma, dn * xh, dn.abs() * e), (dbeta, dn, 0 * dn)):
        want = terms.sum((0, 1))
        tol = err.sum((0, 1)) + (rows + 2) * U * (terms.abs() + err).sum((0, 1))
        assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,M", [("bf16", 512), ("bf16", 8192), ("f32", 20004)])
def test_ds_in_place_of_dres_and_the_same_bits(dtype, M):
    G, S = 2, 150
    d = make(G, S, M, dtype, True)
    sh = moe.MoEShape(G, S, M, M, 2, 1, dtype)
    out = []
    for fill, alias in ((0, False), (0xff, True)):
        ds = d["dres"].clone() if alias else torch.empty_like(d["x"])
        dgamma, dbeta = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        ws = torch.full((moe.moe_layer_norm_backward_workspace_bytes(sh),), fill, dtype=torch.uint8, device=DEV)
        moe.moe_add_layer_norm_backward(sh, d["x"], d["dn"], d["gamma"], ds if alias else d["dres"], ds, dgamma, dbeta, ws)
        out.append((ds, dgamma, dbeta))
    assert all(torch.equal(a, b) for a, b in zip(*out))
