"""Cross attention, the vocabulary's loss, a policy or preference loss on it, their backward passes, the norm and the clipped gradients, as a
program runs them; captured, replayed, on other streams, in guarded buffers and with offsets past 32 bits."""
import pytest
import torch

import paper_2006_16668_amd as moe
from cross_bounds import DT, HALF, U, assert_within, core
from test_gpu_cross_attention import CASES, held, selection

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def nan(*s, dt=torch.float32):
    return torch.full(s, float("nan"), dtype=dt, device=DEV)


class Step:
    """A decoder layer's attention to its sources and the end of the model, tuned on pairs of answers (kind "preference") or sampled ones ("policy")."""
    B, Lq, Lk, M, heads, kv_heads, d, V = 6, 20, 33, 136, 4, 2, 64, 501

    def __init__(self, dtype, kind, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.kind, dt = dtype, kind, DT[dtype]
        B, Lq, Lk, M, V, A, W = self.B, self.Lq, self.Lk, self.M, self.V, self.heads * self.d, 2 * self.kv_heads * self.d
        rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.sh, self.dims, self.vd = moe.MoEShape(B, Lq, M, 64, 2, 1, dtype), moe.CrossDims(B, Lq, Lk, self.heads, self.d, self.kv_heads), moe.VocabDims(V)
        self.pd, self.qd = moe.PreferenceDims(B // 2, V, 0.05, 0.1), moe.PolicyDims(V, 1.0, 1e3, 0.1)
        self.u, self.mem = rand(B, Lq, M).to(dt), rand(B, Lk, M).to(dt)
        self.w = {"wq": rand(M, A) / M ** 0.5, "wkv": rand(M, W) / M ** 0.5, "wo": rand(A, M) / A ** 0.5, "wv": rand(V, M) / M ** 0.5}
        self.w = {k: t.to(dt) for k, t in self.w.items()}
        self.len = torch.randint(1, Lk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        self.target = torch.randint(0, V, (B, Lq), generator=g, device=DEV, dtype=torch.int32)
        self.target[:, :3] = -1
        self.start = torch.arange(0, B * Lq + 1, Lq, dtype=torch.int32, device=DEV)
        self.adv, self.ref = rand(B), 6.2 + 0.3 * rand(B, Lq)
        self.up = (torch.rand(B, Lq, generator=g, device=DEV) + 0.5) / (B * Lq)
        self.pup = (torch.rand(B // 2, generator=g, device=DEV) + 0.5) / (B // 2)
        self.max_norm = 1e-3
        u8 = lambda n: torch.full((n,), 255, dtype=torch.uint8, device=DEV)
        sh = self.sh
        self.fwd, self.bws = u8(moe.moe_cross_train_workspace_bytes(sh, self.dims)), u8(moe.moe_cross_backward_workspace_bytes(sh, self.dims))
        self.vws, self.vbws = u8(moe.moe_vocab_workspace_bytes(sh, self.vd)), u8(moe.moe_vocab_backward_workspace_bytes(sh, self.vd))
        like = torch.empty_like
        self.r = {"kv": nan(B, Lk, W, dt=dt), "out": like(self.u), "nll": nan(B, Lq), "lse": nan(B, Lq), "loss": nan(B // 2) if kind == "preference" else nan(B, Lq),
                  "ratio": nan(B), "dnll": nan(B, Lq), "dout": like(self.u), "du": like(self.u), "dmem": like(self.mem), "norm": nan(1)}
        self.g = {f"d{k}": like(t) for k, t in self.w.items()}
        self.list = moe.GradientList(self.g.values())
        self.nws = u8(moe.moe_gradient_norm_workspace_bytes(self.list))

    def run(self):
        r, w, sh = self.r, self.w, self.sh
        moe.moe_cross_keys(sh, self.dims, self.mem, w["wkv"], r["kv"])
        moe.moe_cross_attention_train(sh, self.dims, self.u, r["kv"], self.len, w["wq"], w["wo"], r["out"], self.fwd)
        moe.moe_vocab_loss(sh, self.vd, r["out"], w["wv"], self.target, r["nll"], r["lse"], self.vws)
        if self.kind == "preference":
            moe.moe_preference_loss(sh, self.pd, r["nll"], self.ref, self.target, self.start, r["loss"], r["ratio"])
            moe.moe_preference_loss_backward(sh, self.pd, self.target, self.start, r["ratio"], self.pup, r["dnll"])
        else:
            moe.moe_policy_loss(sh, self.qd, r["nll"], self.ref, self.ref, self.adv, self.target, r["loss"])
            moe.moe_policy_loss_backward(sh, self.qd, r["nll"], self.ref, self.ref, self.adv, self.target, self.up, r["dnll"])
        moe.moe_vocab_loss_backward(sh, self.vd, r["out"], w["wv"], self.target, r["nll"], r["lse"], r["dnll"], r["dout"], self.g["dwv"], self.vbws)
        grads = {"du": r["du"], "dmem": r["dmem"], **{k: self.g[k] for k in ("dwq", "dwkv", "dwo")}}
        moe.moe_cross_attention_backward(sh, self.dims, self.u, self.mem, r["kv"], self.len, w["wq"], w["wkv"], w["wo"], r["dout"], self.fwd, grads, self.bws)
        moe.moe_gradient_norm(self.list, r["norm"], self.nws)
        moe.moe_clip_gradients(self.list, r["norm"], self.max_norm)
        return {**r, **self.g}

    def reference(self):
        """By automatic differentiation in 64 bits: gradients, their norm, the loss."""
        B, Lq, Lk, d, K, share = self.B, self.Lq, self.Lk, self.d, self.kv_heads, self.heads // self.kv_heads
        leaf = lambda t: t.double().requires_grad_(True)
        u, mem, w = leaf(self.u), leaf(self.mem), {k: leaf(t) for k, t in self.w.items()}
        q = (u @ w["wq"]).view(B, Lq, K, share, d).permute(0, 2, 3, 1, 4)
        kv = (mem @ w["wkv"]).view(B, Lk, 2, K, 1, d).permute(2, 0, 3, 4, 1, 5)
        s = (q[..., :, None, :] * kv[0][..., None, :, :]).sum(-1) / d ** 0.5
        s = s.masked_fill(torch.arange(Lk, device=DEV) >= self.len.view(B, 1, 1, 1, 1), -torch.inf)
        ctx = (torch.softmax(s, -1)[..., None] * kv[1][..., None, :, :]).sum(-2).permute(0, 3, 1, 2, 4).reshape(B, Lq, -1)
        z = (ctx @ w["wo"]) @ w["wv"].t()
        has = self.target >= 0
        nll = torch.logsumexp(z, -1) - z.gather(-1, self.target.clamp(min=0).long()[..., None])[..., 0]
        nll = torch.where(has, nll, 0.0)
        if self.kind == "preference":
            h = torch.where(has, self.ref.double() - nll, 0.0).sum(1)
            x = self.pd.beta * (h[0::2] - h[1::2])
            loss = -(0.9 * torch.nn.functional.logsigmoid(x) + 0.1 * torch.nn.functional.logsigmoid(-x))
            total = (loss * self.pup).sum()
        else:
            r = torch.exp(self.ref.double() - nll)
            x = nll - self.ref.double()
            loss = torch.where(has, -r * self.adv.double()[:, None] + 0.1 * (torch.exp(x) - 1 - x), 0.0)
            total = (loss * self.up).sum()
        total.backward()
        g = {f"d{k}": t.grad for k, t in w.items()}
        norm = sum((t ** 2).sum() for t in g.values()).sqrt()
        scale = min(1.0, self.max_norm / float(norm))
        return {"loss": loss.detach(), "norm": norm.view(1), "du": u.grad, "dmem": mem.grad, **{k: t * scale for k, t in g.items()}}


@pytest.mark.parametrize("kind", ["preference", "policy"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_against_automatic_differentiation(dtype, kind):
    """Ten stored intermediates lie between the inputs and a gradient, each half a step of its elements off, in norm below h; what softmax and
    the losses make of the errors of their inputs (scores and nll below 10) is at most some ten times those."""
    s = Step(dtype, kind)
    got, want = s.run(), s.reference()
    torch.cuda.synchronize()
    h = HALF[dtype] if dtype == "bf16" else 40 * U                # (fp32: sums of a few hundred terms in place of roundings)
    for k, w in want.items():
        err = ((got[k].double() - w).norm() / w.norm()).item()
        assert err < 20 * h, (k, err)
    assert float(want["norm"]) > s.max_norm                      # (so that the clip has something to do)
    clipped = sum((t.double() ** 2).sum() for t in s.g.values()).sqrt().item()
    assert abs(clipped - s.max_norm) < 2 * HALF[dtype] * s.max_norm


@pytest.mark.parametrize("kind", ["preference", "policy"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_step(dtype, kind):
    """Captured once, replayed on new inputs, lengths and targets with eager work between: the eager results, bit for bit."""
    moe.moe_prepare()
    s = Step(dtype, kind)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for i in range(4):
        e = Step(dtype, kind, seed=i)
        if i == 2:
            e.len[1] = 0
            e.target[0, :] = -1
        for a, b in ((s.u, e.u), (s.mem, e.mem), (s.len, e.len), (s.target, e.target), (s.adv, e.adv), (s.ref, e.ref), (s.up, e.up), (s.pup, e.pup)):
            a.copy_(b)
        for k in s.w:
            s.w[k].copy_(e.w[k])
        want = {k: v.clone() for k, v in e.run().items() if not (kind == "policy" and k == "ratio")}
        for t in list(s.r.values()) + list(s.g.values()):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = {**s.r, **s.g}
        for k, v in want.items():
            assert torch.equal(got[k], v), (i, k)


def cross_call(c, dtype, seed=0, ws_fill=255):
    """Inputs, and a function that runs all of a layer's calls in buffers of its own and gives what they left."""
    B, Lq, Lk, heads, kv_heads, d, kind = c
    g = torch.Generator(device=DEV).manual_seed(seed + B + Lk)
    dt, M, A, W = DT[dtype], 72, heads * d, 2 * kv_heads * d
    sh, dims = moe.MoEShape(B, Lq, M, 64, 2, 1, dtype), moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dt)
    u, mem, dout, wq, wkv, wo = rand(B, Lq, M), rand(B, Lk, M), rand(B, Lq, M), rand(M, A) / 8, rand(M, W) / 8, rand(A, M) / 16
    src = torch.randint(0, Lk + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if kind else None
    need = (moe.moe_cross_workspace_bytes(sh, dims), moe.moe_cross_train_workspace_bytes(sh, dims), moe.moe_cross_backward_workspace_bytes(sh, dims))

    def run(ws=None):
        ws = ws or [torch.full((n,), ws_fill, dtype=torch.uint8, device=DEV) for n in need]
        kv, out, train = nan(B, Lk, W, dt=dt), nan(B, Lq, M, dt=dt), nan(B, Lq, M, dt=dt)
        grads = {"du": nan(B, Lq, M, dt=dt), "dmem": nan(B, Lk, M, dt=dt), "dwq": nan(M, A, dt=dt), "dwkv": nan(M, W, dt=dt), "dwo": nan(A, M, dt=dt)}
        moe.moe_cross_keys(sh, dims, mem, wkv, kv)
        moe.moe_cross_attention(sh, dims, u, kv, src, wq, wo, out, ws[0])
        moe.moe_cross_attention_train(sh, dims, u, kv, src, wq, wo, train, ws[1])
        moe.moe_cross_attention_backward(sh, dims, u, mem, kv, src, wq, wkv, wo, dout, ws[1], grads, ws[2])
        return {"kv": kv, "out": out, "train": train, **grads}

    return need, run


FORMS = [(3, 200, 300, 4, 2, 64, "any"), (1, 300, 1000, 2, 2, 128, "any"), (2, 1, 4100, 2, 2, 128, "any"), (40, 70, 200, 8, 8, 128, "any"), (9, 5, 700, 16, 2, 64, None),
         (2, 1500, 70, 4, 1, 64, "any")]                  # dK and dV in ranges of columns


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", FORMS)
def test_same_bits_whatever_the_workspace_held(c, dtype):
    want = cross_call(c, dtype, ws_fill=255)[1]()
    for fill in (0, 0x3f, 255):
        got = cross_call(c, dtype, ws_fill=fill)[1]()
        for k, v in want.items():
            assert torch.equal(got[k], v), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_graphs_share_workspaces(dtype):
    """Each call leaves nothing in its workspace that another needs (but for the backward pass's own forward): graphs of different sizes in turn."""
    moe.moe_prepare()
    jobs = [cross_call(c, dtype) for c in FORMS[:4] + FORMS[5:]]
    ws = [torch.full((max(j[0][i] for j in jobs),), 255, dtype=torch.uint8, device=DEV) for i in range(3)]
    wants = [run() for _, run in jobs]
    graphs = []
    for _, run in jobs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run(ws)
        graphs.append((graph, out))
    for turn in (0, 1, 2, 3, 4, 3, 1, 4, 0, 2):
        graph, out = graphs[turn]
        graph.replay()
        torch.cuda.synchronize()
        for k, v in wants[turn].items():
            assert torch.equal(out[k], v), (turn, k)


@pytest.mark.parametrize("one,other,dtype", [(FORMS[0], FORMS[2], "bf16"), (FORMS[3], FORMS[1], "bf16"), (FORMS[5], FORMS[0], "bf16"), (FORMS[0], FORMS[3], "f32"), (FORMS[2], FORMS[4], "f32")])
def test_streams_that_run_at_once(one, other, dtype):
    """All enqueued on two streams before the first may start: kernels of one call run beside kernels of the other."""
    moe.moe_prepare()
    jobs = [cross_call(one, dtype, seed=5), cross_call(other, dtype, seed=6)]
    wants, streams, got = [run() for _, run in jobs], [torch.cuda.Stream() for _ in jobs], [[], []]
    torch.cuda.synchronize()
    start = torch.cuda.Event()
    torch.cuda._sleep(60_000_000)
    start.record()
    for st in streams:
        st.wait_event(start)
    for _ in range(3):
        for i, (_, run) in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                got[i].append(run())
    torch.cuda.synchronize()
    for i, results in enumerate(got):
        for r in results:
            for k, v in wants[i].items():
                assert torch.equal(r[k], v), (i, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", [CASES[2], CASES[3], CASES[5], CASES[8], CASES[11], CASES[12], CASES[17]])
def test_nothing_is_written_outside(c, dtype):
    """Outputs and workspaces of exactly their size between guards."""
    B, Lq, Lk, heads, kv_heads, d, _ = c
    g = torch.Generator(device=DEV).manual_seed(1)
    dt, M, A, W = DT[dtype], 40, heads * d, 2 * kv_heads * d
    sh, dims = moe.MoEShape(B, Lq, M, 64, 2, 1, dtype), moe.CrossDims(B, Lq, Lk, heads, d, kv_heads)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dt)
    guarded = []

    def guard(shape, t):
        n = int(torch.tensor(shape).prod())
        pad = 4096 // torch.empty(0, dtype=t).element_size()
        buf = torch.full((n + 2 * pad,), 77, dtype=t, device=DEV)
        guarded.append((buf, pad, n))
        return buf[pad:pad + n].view(shape)

    u, mem, dout, wq, wkv, wo = rand(B, Lq, M), rand(B, Lk, M), rand(B, Lq, M), rand(M, A), rand(M, W), rand(A, M)
    src = torch.randint(0, Lk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    inputs = [t.clone() for t in (u, mem, dout, wq, wkv, wo, src)]
    kv, out = guard((B, Lk, W), dt), guard((B, Lq, M), dt)
    ws = [guard((n,), torch.uint8) for n in (moe.moe_cross_workspace_bytes(sh, dims), moe.moe_cross_train_workspace_bytes(sh, dims),
                                             moe.moe_cross_backward_workspace_bytes(sh, dims))]
    grads = {"du": guard((B, Lq, M), dt), "dmem": guard((B, Lk, M), dt), "dwq": guard((M, A), dt), "dwkv": guard((M, W), dt), "dwo": guard((A, M), dt)}
    moe.moe_cross_keys(sh, dims, mem, wkv, kv)
    moe.moe_cross_attention(sh, dims, u, kv, src, wq, wo, out, ws[0])
    moe.moe_cross_attention_train(sh, dims, u, kv, src, wq, wo, out, ws[1])
    kept = kv.clone(), ws[1].clone()
    moe.moe_cross_attention_backward(sh, dims, u, mem, kv, src, wq, wkv, wo, dout, ws[1], grads, ws[2])
    torch.cuda.synchronize()
    for buf, pad, n in guarded:
        assert (buf[:pad] == 77).all() and (buf[pad + n:] == 77).all()
    assert torch.equal(kv, kept[0]) and torch.equal(ws[1], kept[1])
    for a, b in zip((u, mem, dout, wq, wkv, wo, src), inputs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,Lq,Lk", [("bf16", 1, 600_001), ("bf16", 40, 600_001), ("bf16", 130, 300_033), ("f32", 1, 300_017), ("f32", 33, 270_001)])
def test_states_past_4_gb(dtype, Lq, Lk):
    """16 heads of 128: rows of K and V lie 8 KB (fp32 16 KB) apart.  Every score but those of the last 64 states is so low that they alone
    count; their gradients too are what 64 states by themselves give."""
    g = torch.Generator(device=DEV).manual_seed(9)
    B, heads, d, dt = (2 if Lq > 100 else 1), 16, 128, DT[dtype]
    A = heads * d
    M, tail = 2 * A, 64
    dims = moe.CrossDims(B, Lq, Lk, heads, d)
    sh = moe.MoEShape(B, Lq, M, 64, 2, 1, dtype)
    assert B * Lk * 2 * A * torch.empty(0, dtype=dt).element_size() > 1 << 32
    u = torch.randn(B, Lq, M, generator=g, device=DEV).to(dt)
    u[..., 0:A:d] = 100.0                                        # the first d of every head
    kv = torch.zeros(B, Lk, 2 * A, dtype=dt, device=DEV)
    kv[..., 0:A:d] = -40.0                                       # scores of -350
    kv[:, -tail:] = torch.randn(B, tail, 2 * A, generator=g, device=DEV).to(dt)
    kv[:, -tail:, 0:A:d] = 0.0
    w = (selection(M, A, dt), selection(A, M, dt))
    out = nan(B, Lq, M, dt=dt)
    u8 = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    fwd = u8(moe.moe_cross_train_workspace_bytes(sh, dims))
    moe.moe_cross_attention_train(sh, dims, u, kv, None, w[0], w[1], out, fwd)
    dout = torch.randn(B, Lq, M, generator=g, device=DEV).to(dt)
    ref = core(u[..., :A], kv[:, -tail:], [tail] * B, heads, 1, d, dtype, dout[..., :A])
    # (the others' probabilities are below e^-300; sums in ranges of states add as many roundings as there are ranges)
    extra = 1 + 64 * U / HALF[dtype]
    assert_within(out[..., :A], ref["ctx"][0], extra * ref["ctx"][1], "ctx")
    wkv = selection(M, 2 * A, dt)
    mem = kv                                                     # (as wide, and so selected)
    grads = {"du": nan(B, Lq, M, dt=dt), "dmem": nan(B, Lk, M, dt=dt), "dwq": nan(M, A, dt=dt), "dwkv": nan(M, 2 * A, dt=dt), "dwo": nan(A, M, dt=dt)}
    moe.moe_cross_attention_backward(sh, dims, u, mem, kv, None, w[0], wkv, w[1], dout, fwd, grads, u8(moe.moe_cross_backward_workspace_bytes(sh, dims)))
    assert_within(grads["du"][..., :A], ref["dq"][0], extra * ref["dq"][1], "dq")
    assert_within(grads["dmem"][:, -tail:], ref["dkv"][0], extra * ref["dkv"][1], "dkv")
    assert (grads["dmem"][:, :-tail] == 0).all()
