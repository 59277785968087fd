"""Cross attention against its formulas in 64 bits.

The attention itself is looked at through projections that only select columns (products with 1 and 0 and their sums are exact), so that
every element of ctx, dq, dK and dV has the bounds derived in cross_bounds.py; the layer with its projections has those and the
projections' own roundings."""
import math

import pytest
import torch

import paper_2006_16668_amd as moe
from cross_bounds import DT, HALF, U, assert_within, core

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def selection(rows, cols, dt):
    w = torch.zeros(rows, cols, dtype=dt, device=DEV)
    w.fill_diagonal_(1.0)
    return w


def _bytes(n):
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV)           # (NaN as fp32 and as bf16)


def _rand(g, *s, dt):
    return torch.randn(*s, generator=g, device=DEV).to(dt)


def run(dims, dtype, u, mem, kv, src_len, wq, wkv, wo, dout=None):
    """out, and with dout the gradients."""
    sh = moe.MoEShape(dims.B, dims.Lq, u.shape[2], 64, 2, 1, dtype)
    out = torch.full_like(u, float("nan"))
    if dout is None:
        moe.moe_cross_attention(sh, dims, u, kv, src_len, wq, wo, out, _bytes(moe.moe_cross_workspace_bytes(sh, dims)))
        return out, None
    fwd = _bytes(moe.moe_cross_train_workspace_bytes(sh, dims))
    moe.moe_cross_attention_train(sh, dims, u, kv, src_len, wq, wo, out, fwd)
    grads = {k: torch.full_like(t, float("nan")) for k, t in (("du", u), ("dmem", mem), ("dwq", wq), ("dwkv", wkv), ("dwo", wo))}
    moe.moe_cross_attention_backward(sh, dims, u, mem, kv, src_len, wq, wkv, wo, dout, fwd, grads,
                                     _bytes(moe.moe_cross_backward_workspace_bytes(sh, dims)))
    return out, grads


def lens(B, Lk, kind, g):
    if kind is None:
        return None
    if kind == "ends":                        # one state, none, all, all but one, more and fewer than there can be
        n = [1, 0, Lk, Lk - 1, Lk + 5, -3]
        return torch.tensor([n[i % 6] for i in range(B)], dtype=torch.int32, device=DEV)
    return torch.randint(0, Lk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)


def held(src_len, B, Lk):
    return [Lk] * B if src_len is None else [min(max(int(v), 0), Lk) for v in src_len.tolist()]


# B, Lq, Lk, heads, kv_heads, d, lengths
CASES = [(1, 1, 1, 1, 1, 64, None), (6, 1, 1, 2, 2, 128, "ends"), (4, 40, 1, 4, 2, 64, None), (7, 3, 9, 2, 1, 128, "ends"), (3, 150, 31, 2, 2, 64, "ends"), (6, 3, 64, 2, 1, 64, "ends"), (6, 33, 65, 2, 2, 128, "ends"),
         (6, 31, 129, 4, 1, 64, "ends"), (3, 128, 128, 2, 2, 128, None), (2, 129, 63, 8, 1, 128, "any"), (3, 200, 300, 4, 2, 64, "any"),
         (1, 300, 1000, 2, 2, 128, "any"), (5, 64, 257, 4, 4, 64, None), (2, 1, 4100, 2, 2, 128, "any"), (9, 5, 700, 16, 2, 64, "any"),
         (2, 1, 333, 32, 1, 64, "any"), (1, 515, 77, 2, 2, 64, None), (1, 1, 2000, 1, 1, 128, None), (40, 2, 190, 3, 3, 64, "any"),
         (130, 130, 70, 2, 2, 128, "any"),
         # two tiles of states a wavefront backward; as many ranges of states as there are; ranges, some of which a short source leaves empty
         (40, 70, 200, 8, 8, 128, "any"), (1, 2, 8200, 1, 1, 64, None), (6, 4, 2500, 1, 1, 128, "ends"), (70, 31, 33, 4, 4, 128, "any"),
         (2, 500, 890, 8, 8, 64, "any"), (1, 500, 500, 8, 8, 128, "any"),
         # dq in blocks of 128 columns: more blocks of 32 than the units take at once, with each end of the states
         (33, 100, 130, 4, 4, 64, "ends"), (24, 100, 97, 4, 4, 128, "ends"), (33, 17, 130, 8, 4, 64, "ends"), (66, 40, 193, 4, 1, 128, "ends"),
         # and as many as they take
         (16, 63, 256, 8, 8, 128, "ends"), (2, 1000, 100, 8, 8, 64, "ends"),
         # dK and dV in ranges of columns: whole ones, a last one that is shorter, whose last block is not whole, sources of every length
         (1, 1024, 60, 2, 2, 128, None), (6, 900, 130, 4, 4, 64, "ends"), (7, 401, 70, 2, 1, 128, "ends"), (2, 777, 300, 4, 1, 64, "any")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Lq,Lk,heads,kv_heads,d,kind", CASES)
def test_attention_and_its_gradients(dtype, B, Lq, Lk, heads, kv_heads, d, kind):
    g = torch.Generator(device=DEV).manual_seed(B * 7 + Lq * 11 + Lk * 13 + heads)
    dt, A, W = DT[dtype], heads * d, 2 * kv_heads * d
    M = max(A, W)
    dims = moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    print(f"case {dims} {dtype}", flush=True)
    src_len = lens(B, Lk, kind, g)
    n = held(src_len, B, Lk)
    u, kv, dout = _rand(g, B, Lq, M, dt=dt), _rand(g, B, Lk, W, dt=dt), _rand(g, B, Lq, M, dt=dt)
    u[..., :A] *= 1.5
    mem = torch.zeros(B, Lk, M, dtype=dt, device=DEV)
    mem[..., :W] = kv
    for b in range(B):                        # whatever stands behind the last state has no part
        kv[b, n[b]:] = float("nan")
        mem[b, n[b]:] = float("inf")
    out, grads = run(dims, dtype, u, mem, kv, src_len, selection(M, A, dt), selection(M, W, dt), selection(A, M, dt), dout)
    inferred, _ = run(dims, dtype, u, mem, kv, src_len, selection(M, A, dt), selection(M, W, dt), selection(A, M, dt))
    assert torch.equal(inferred, out)
    ref = core(u[..., :A], kv, n, kv_heads, heads // kv_heads, d, dtype, dout[..., :A])
    assert_within(out[..., :A], *ref["ctx"], "ctx")
    assert_within(grads["du"][..., :A], *ref["dq"], "dq")
    assert_within(grads["dmem"][..., :W], *ref["dkv"], "dkv")
    for t, c in ((out, A), (grads["du"], A), (grads["dmem"], W)):
        assert (t[..., c:] == 0).all()
    for b in range(B):
        assert (grads["dmem"][b, n[b]:] == 0).all()
        if n[b] == 0:
            assert (out[b] == 0).all() and (grads["du"][b] == 0).all()
        if n[b] == 1 and Lk <= 32:            # one state has a probability of 1 whatever the query: nothing passes to it, to the last bit
            assert (grads["du"][b] == 0).all()


@pytest.mark.parametrize("dtype,B,Lq,Lk,M,heads,kv_heads,d,kind", [
    ("bf16", 3, 70, 150, 264, 4, 2, 64, "any"), ("f32", 3, 70, 150, 260, 4, 4, 64, "any"), ("bf16", 7, 1, 90, 512, 4, 4, 128, None),
    ("f32", 2, 2, 333, 132, 2, 1, 128, "any"), ("f32", 2, 5, 7, 1284, 4, 2, 64, "any"), ("f32", 1, 1, 1, 4, 1, 1, 64, None), ("bf16", 1, 1, 1, 8, 1, 1, 64, None),
    ("bf16", 2, 200, 130, 1024, 8, 8, 64, None)])
def test_layer_with_its_projections(dtype, B, Lq, Lk, M, heads, kv_heads, d, kind):
    g = torch.Generator(device=DEV).manual_seed(M + Lk)
    dt, h, A, W = DT[dtype], HALF[dtype], heads * d, 2 * kv_heads * d
    dims = moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    sh = moe.MoEShape(B, Lq, M, 64, 2, 1, dtype)
    src_len = lens(B, Lk, kind, g)
    n = held(src_len, B, Lk)
    u, mem, dout = _rand(g, B, Lq, M, dt=dt), _rand(g, B, Lk, M, dt=dt), _rand(g, B, Lq, M, dt=dt)
    wq, wkv, wo = ((_rand(g, *s, dt=torch.float32) / s[0] ** 0.5).to(dt) for s in ((M, A), (M, W), (A, M)))
    kv = torch.full((B, Lk, W), float("nan"), dtype=dt, device=DEV)
    moe.moe_cross_keys(sh, dims, mem, wkv, kv)
    D = lambda t: t.double()
    prod = lambda a, b, k: (a @ b, (h * (a @ b).abs() + 2 * k * max(U, 0) * (a.abs() @ b.abs())))
    assert_within(kv, *prod(D(mem), D(wkv), M), "kv")
    out, grads = run(dims, dtype, u, mem, kv, src_len, wq, wkv, wo, dout)
    q, e_q = prod(D(u), D(wq), M)
    dctx, e_dctx = prod(D(dout), D(wo).t(), M)
    ref = core(q, kv, n, kv_heads, heads // kv_heads, d, dtype, dctx, e_q)
    ctx, e_ctx = ref["ctx"]
    want = ctx @ D(wo)
    assert_within(out, want, e_ctx @ D(wo).abs() + 2 * A * U * (ctx.abs() @ D(wo).abs()) + h * want.abs(), "out")
    # gradients: what dctx's rounding adds is as large again as a dctx of its size gives (they are linear in dctx), with e_dctx <= e |dctx|'s rows
    rel = float((e_dctx.norm() / dctx.norm()))
    flat = lambda t: t.reshape(-1, t.shape[-1])
    norms = {"du": (ref["dq"][0] @ D(wq).t(), ref["dq"][1] @ D(wq).abs().t()),
             "dmem": (ref["dkv"][0] @ D(wkv).t(), ref["dkv"][1] @ D(wkv).abs().t()),
             "dwq": (flat(D(u)).t() @ flat(ref["dq"][0]), flat(D(u)).abs().t() @ flat(ref["dq"][1])),
             "dwkv": (flat(D(mem)).t() @ flat(ref["dkv"][0]), flat(D(mem)).abs().t() @ flat(ref["dkv"][1])),
             "dwo": (flat(ctx).t() @ flat(D(dout)), flat(e_ctx).t() @ flat(D(dout)).abs())}
    for name, (want, err) in norms.items():
        got = D(grads[name])
        assert torch.isfinite(got).all(), name
        bound = err.norm() + (3 * rel + 2 * h + 2 * max(M, A, B * Lq, B * Lk) * U) * want.norm()
        assert (got - want).norm() <= bound, (name, float((got - want).norm() / want.norm()), float(bound / want.norm()))
        # and not only within the worst case: roundings of independent sign leave a few h.  (One state: p = 1 and dS = 0, and what the 64-bit sums leave
        # of it is their own rounding, n 2^-53 of magnitudes of which err has at least 2^-24: n 2^-29 err, below 2^-20 err for sums of 512 terms.)
        assert (got - want).norm() <= (6 * h + 2000 * U) * want.norm() + 2.0 ** -20 * err.norm(), (name, float((got - want).norm() / want.norm()))


def test_gradients_against_differences():
    """Central differences of the 64-bit forward pass: the formulas that the other tests compare with are the derivative."""
    g = torch.Generator(device=DEV).manual_seed(3)
    B, Lq, Lk, K, share, d = 2, 3, 5, 2, 2, 64
    q, kv, dctx = (torch.randn(*s, generator=g, device=DEV, dtype=torch.float64) for s in ((B, Lq, K * share * d), (B, Lk, 2 * K * d), (B, Lq, K * share * d)))
    n = [5, 3]
    f = lambda q, kv: float((core(q, kv, n, K, share, d, "f32")["ctx"][0] * dctx).sum())
    ref = core(q, kv, n, K, share, d, "f32", dctx)
    for t, name in ((q, "dq"), (kv, "dkv")):
        for _ in range(5):
            at = tuple(int(torch.randint(0, s, (1,), generator=g, device=DEV)) for s in t.shape)
            step = torch.zeros_like(t)
            step[at] = 1e-5
            a = (q + step, kv) if t is q else (q, kv + step)
            b = (q - step, kv) if t is q else (q, kv - step)
            want = float(ref[name][0][at])
            assert math.isclose((f(*a) - f(*b)) / 2e-5, want, rel_tol=1e-5, abs_tol=1e-8)


@pytest.mark.parametrize("rows,M,heads", [(1, 8, 1), (1, 1024, 8), (3, 72, 2), (31, 520, 1), (32, 64, 3), (33, 2056, 1), (64, 1000, 8), (65, 264, 2),
                                          (128, 1024, 16), (256, 128, 4), (257, 136, 1), (2048, 40, 1), (2049, 40, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_of_few_and_more_rows(rows, M, heads, dtype):
    """Products whose tiles of 32 x 32 fill the device once, and larger ones: sums of 8 to 2056 terms, ends inside a tile, a chunk, a piece."""
    g = torch.Generator(device=DEV).manual_seed(rows + M)
    W = 2 * heads * 64
    mem, wkv = _rand(g, 1, rows, M, dt=DT[dtype]), _rand(g, M, W, dt=DT[dtype])
    room = torch.full((rows * W + 256,), 7.0, dtype=DT[dtype], device=DEV)
    kv = room[128:128 + rows * W].view(1, rows, W)
    moe.moe_cross_keys(moe.MoEShape(1, 1, M, 64, 2, 1, dtype), moe.CrossDims(1, 1, rows, heads, 64), mem, wkv, kv)
    want, size = mem.double() @ wkv.double(), mem.double().abs() @ wkv.double().abs()
    assert_within(kv, want, HALF[dtype] * want.abs() + M * U * size, "kv")
    assert (room[:128] == 7).all() and (room[-128:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Lk", [2, 3, 31, 33, 64, 65])
def test_gradients_of_few_states(Lk, dtype):
    """dP - D is a difference of near numbers where states are few.  D comes from the probabilities at hand up to 64 (fp32: 32) states, and dq in norm is then off
    by the roundings of dS and of itself, a third of h each in the mean (h / sqrt(12) 2 for numbers spread over a binade), not by that of a stored ctx."""
    g = torch.Generator(device=DEV).manual_seed(Lk)
    B, Lq, heads, d, dt = 4, 65, 2, 64, DT[dtype]
    A = heads * d
    M = 2 * A
    u, kv, dout = (_rand(g, B, n, M, dt=dt) for n in (Lq, Lk, Lq))
    w = selection(M, A, dt), selection(M, M, dt), selection(A, M, dt)
    out, grads = run(moe.CrossDims(B, Lq, Lk, heads, d), dtype, u, kv.clone(), kv, None, *w, dout)
    ref = core(u[..., :A], kv, [Lk] * B, heads, 1, d, dtype, dout[..., :A])
    err = (grads["du"][..., :A].double() - ref["dq"][0]).norm() / ref["dq"][0].norm()
    assert err < (0.85 if dtype == "bf16" and Lk <= 64 else 1.2 if dtype == "bf16" else 12) * HALF[dtype], float(err / HALF[dtype])
