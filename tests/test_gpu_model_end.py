"""The end of a model as a training step uses it: encoder layers, final normalisation, both losses over the vocabulary, and back; in
graphs, on other streams, with shared workspaces.
"""
import pytest
import torch

import paper_2006_16668_amd as moe
from harness import shape_of
from oracle import transformer_oracle_backward as trb
from oracle import vocab_oracle as orc
from test_gpu_vocab_loss import DT, call, make
from workloads import MoEConfig, make_encoder_weights, make_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Step:
    """One training step of a small model; all buffers its own."""

    def __init__(self, dtype, V=203, K=5):
        self.cfg = MoEConfig("model_end", G=2, S=60, M=64, H=128, E=4, C=40, act_dtype=dtype, seed=77)
        self.sh, self.dims = shape_of(self.cfg), moe.EncoderDims(4, 30, 2, 32)
        self.ce, self.kd = moe.VocabDims(V), moe.VocabDims(V, K=K, temperature=2.0)
        self.inp = make_inputs(self.cfg, device=DEV)
        self.w = dict(make_encoder_weights(self.cfg, 2, 32, device=DEV), wg=self.inp.wg, wi=self.inp.wi, wo=self.inp.wo)
        G, S, M = self.cfg.G, self.cfg.S, self.cfg.M
        g = torch.Generator(device=DEV).manual_seed(5)
        rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.gamma, self.beta = 1 + 0.1 * rand(M), 0.1 * rand(M)
        self.out = (rand(V, M) / 8).to(DT[dtype])
        self.target = torch.randint(0, V, (G, S), generator=g, device=DEV).int()
        self.target[:, ::7] = -1
        self.idx = torch.randint(0, V, (G, S, K), generator=g, device=DEV).int()
        self.idx[0, :9] = -1
        self.logit = 2 * rand(G, S, K)
        self.dloss = [torch.rand(G, S, generator=g, device=DEV) / (G * S) for _ in range(2)]
        self.daux = torch.rand(G, generator=g, device=DEV)
        self.r = None

    def forward(self, x):
        G, S, M, K = self.cfg.G, self.cfg.S, self.cfg.M, self.kd.K
        e = torch.empty
        if self.r is None:
            u8 = lambda n: e(n, dtype=torch.uint8, device=DEV)
            f = lambda *s: e(*s, device=DEV)
            sh = self.sh
            self.r = {"y": e(G, S, M, dtype=DT[self.cfg.act_dtype], device=DEV), "n": e(G, S, M, dtype=DT[self.cfg.act_dtype], device=DEV),
                      "aux": f(G), "ce": f(G, S), "ce_lse": f(G, S), "kd": f(G, S), "kd_lse": f(G, S), "entry": f(G, S, K),
                      "fws": u8(moe.moe_encoder_train_workspace_bytes(sh, self.dims)),
                      "bws": u8(moe.moe_encoder_backward_workspace_bytes(sh, self.dims)),
                      "vws": u8(max(moe.moe_vocab_workspace_bytes(sh, d) for d in (self.ce, self.kd))),
                      "vbws": u8(max(moe.moe_vocab_backward_workspace_bytes(sh, d) for d in (self.ce, self.kd))),
                      "lws": u8(moe.moe_layer_norm_backward_workspace_bytes(sh))}
        r = self.r
        moe.moe_encoder_pair_forward_train(self.sh, self.dims, x, self.w, self.inp.u, r["y"], r["aux"], r["fws"])
        moe.moe_add_layer_norm(self.sh, r["y"], None, self.gamma, self.beta, None, r["n"])
        moe.moe_vocab_loss(self.sh, self.ce, r["n"], self.out, self.target, r["ce"], r["ce_lse"], r["vws"])
        moe.moe_vocab_distill(self.sh, self.kd, r["n"], self.out, self.idx, self.logit, r["kd"], r["kd_lse"], r["entry"], r["vws"])
        return r

    def loss(self, x):
        r = self.forward(x)
        return ((r["ce"].double() * self.dloss[0]).sum() + (r["kd"].double() * self.dloss[1]).sum() +
                (r["aux"].double() * self.daux).sum()).item()

    def backward(self, x):
        r, like = self.r, torch.empty_like
        if "dx" not in r:
            r.update(dn1=like(r["n"]), dn2=like(r["n"]), dn=like(r["n"]), dw1=like(self.out), dw2=like(self.out), dy=like(r["y"]),
                     dgamma=like(self.gamma), dbeta=like(self.beta), dx=like(x),
                     grads={k: [like(t) for t in v] if isinstance(v, (list, tuple)) else like(v) for k, v in self.w.items()})
        moe.moe_vocab_loss_backward(self.sh, self.ce, r["n"], self.out, self.target, r["ce"], r["ce_lse"], self.dloss[0], r["dn1"],
                                    r["dw1"], r["vbws"])
        moe.moe_vocab_distill_backward(self.sh, self.kd, r["n"], self.out, self.idx, self.logit, r["entry"], r["kd_lse"], self.dloss[1],
                                       r["dn2"], r["dw2"], r["vbws"])
        torch.add(r["dn1"], r["dn2"], out=r["dn"])
        moe.moe_add_layer_norm_backward(self.sh, r["y"], r["dn"], self.gamma, None, r["dy"], r["dgamma"], r["dbeta"], r["lws"])
        moe.moe_encoder_pair_backward(self.sh, self.dims, x, self.w, r["dy"], self.daux, r["fws"], r["dx"], r["grads"], r["bws"])
        return r

    KEYS = ("ce", "kd", "entry", "dn1", "dn2", "dw1", "dw2", "dy", "dgamma", "dbeta", "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_step_against_the_formulas(dtype):
    """Every stage at its own inputs; norms, so the tolerance counts roundings: half steps of outputs and of dz (bf16 2^-8 each),
    fp32 sums of up to 203 terms (64 . 2 u for products of 64)."""
    s = Step(dtype)
    s.forward(s.inp.x)
    r = s.backward(s.inp.x)
    torch.cuda.synchronize()
    M, V = s.cfg.M, s.ce.V
    n, tol = r["n"].view(-1, M), {"f32": 1e-5, "bf16": 2 * 2.0 ** -8}[dtype]
    rel = lambda a, b: ((a.double() - b).norm() / b.norm()).item()
    q, has = orc.target_weights(n.shape[0], V, s.target.view(-1), DEV)
    dx, dw, _ = orc.backward(n, s.out, s.dloss[0].view(-1), q, has)
    loss, _ = orc.cross_entropy(n, s.out, s.target.view(-1))
    assert rel(r["ce"].view(-1), loss) < 1e-5 and rel(r["dn1"].view(-1, M), dx) < tol and rel(r["dw1"], dw) < tol
    q, has, _, _ = orc.teacher_weights(n.shape[0], V, s.idx.view(-1, 5), s.logit.view(-1, 5), 2.0, DEV)
    dx, dw, _ = orc.backward(n, s.out, s.dloss[1].view(-1), q, has, 2.0)
    loss, _, _ = orc.distill(n, s.out, s.idx.view(-1, 5), s.logit.view(-1, 5), 2.0)
    assert rel(r["kd"].view(-1), loss) < 1e-5 and rel(r["dn2"].view(-1, M), dx) < tol and rel(r["dw2"], dw) < tol
    f64 = lambda t: t.double().cpu().numpy()
    dy, dgamma, dbeta = (torch.from_numpy(t).to(DEV) for t in trb.layer_norm_backward(f64(r["y"]), f64(s.gamma), f64(r["dn"])))
    assert rel(r["dy"], dy) < tol and rel(r["dgamma"], dgamma) < 1e-5 and rel(r["dbeta"], dbeta) < 1e-5


def test_training_step_by_differences():
    """fp32: the loss of the whole model along its gradient.  Its value, about 8, is rounded to 2^-24 in a few hundred places of random sign:
    2e-6 over a step of 2 h |dx| = 2e-3 in x; the routing's decisions have margins larger than the step."""
    s = Step("f32")
    x = s.inp.x.clone()
    s.loss(x)
    dx = s.backward(x)["dx"].double()
    torch.cuda.synchronize()
    v = dx / dx.norm()
    h = 0.1
    # the direction is spread over 7680 numbers: none moves by more than 0.1 of 1
    up, down = (s.loss((x.double() + sign * h * v).float()) for sign in (1, -1))
    assert abs((up - down) / (2 * h) - dx.norm().item()) < 0.02 * dx.norm().item()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_of_a_training_step(dtype):
    """Captured once, replayed on new inputs with eager work between: the eager results, bit for bit."""
    moe.moe_prepare()
    s, eager = Step(dtype), Step(dtype)
    x = s.inp.x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.forward(x)
        s.backward(x)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.forward(x)
        s.backward(x)
    for i in range(4):
        x.copy_(s.inp.x.float() * (1 + 0.01 * i))
        s.target.copy_(torch.where(torch.arange(60, device=DEV) % (i + 2) == 0, -1, eager.target))
        s.idx[1, :20 * i] = -1
        eager_s = Step(dtype)
        eager_s.target.copy_(s.target)
        eager_s.idx.copy_(s.idx)
        eager_s.forward(x)
        want = {k: eager_s.backward(x)[k].clone() for k in Step.KEYS}
        for k in Step.KEYS:
            s.r[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in Step.KEYS:
            assert torch.equal(s.r[k], want[k]), (i, k)


CASES = [(1, 40, 64, 700, "bf16", 0), (1, 40, 64, 700, "f32", 3), (1, 1500, 1024, 9001, "bf16", 0), (1, 2100, 768, 17000, "bf16", 32)]


@pytest.mark.parametrize("G,S,M,V,dtype,K", CASES)
def test_two_graphs_share_a_workspace(G, S, M, V, dtype, K):
    """Each call leaves nothing in its workspace that another needs: graphs of different sizes replayed in turn on one."""
    moe.moe_prepare()
    jobs, need = [], 0
    for s in (S, S // 2 + 1):
        d = make(G, s, M, V, dtype, 0.2, K)
        want = call(G, s, M, V, dtype, d, K, 2.0)
        sh, dims = moe.MoEShape(G, s, M, M, 2, 1, dtype), moe.VocabDims(V, K=K, temperature=2.0)
        need = max(need, moe.moe_vocab_workspace_bytes(sh, dims), moe.moe_vocab_backward_workspace_bytes(sh, dims))
        jobs.append((d, want, sh, dims, s))
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    graphs = []
    for d, want, sh, dims, s in jobs:
        x, f = d["x"].view(G, s, M), lambda *a: torch.full(a, float("nan"), device=DEV)
        out = {"loss": f(G, s), "lse": f(G, s), "dx": torch.full_like(x, float("nan")), "dw": torch.full_like(d["w"], float("nan"))}
        if K:
            out["entry_logit"] = f(G, s, K)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if K:
                idx, logit = d["idx"].view(G, s, K), d["logit"].view(G, s, K)
                moe.moe_vocab_distill(sh, dims, x, d["w"], idx, logit, out["loss"], out["lse"], out["entry_logit"], ws)
                moe.moe_vocab_distill_backward(sh, dims, x, d["w"], idx, logit, out["entry_logit"], out["lse"],
                                               d["dloss"].view(G, s), out["dx"], out["dw"], ws)
            else:
                t = d["target"].view(G, s)
                moe.moe_vocab_loss(sh, dims, x, d["w"], t, out["loss"], out["lse"], ws)
                moe.moe_vocab_loss_backward(sh, dims, x, d["w"], t, out["loss"], out["lse"], d["dloss"].view(G, s), out["dx"],
                                            out["dw"], ws)
        graphs.append((graph, out, want))
    for turn in (0, 1, 1, 0, 1):
        graph, out, want = graphs[turn]
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for k, t in out.items():
            assert torch.equal(t.view(want[k].shape), want[k]), (turn, k)


@pytest.mark.parametrize("G,S,M,V,dtype,K", CASES)
def test_two_streams_at_once(G, S, M, V, dtype, K):
    d = make(G, S, M, V, dtype, 0.2, K)
    want = call(G, S, M, V, dtype, d, K, 2.0)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for st in streams:
        with torch.cuda.stream(st):
            got.append(call(G, S, M, V, dtype, d, K, 2.0))
    torch.cuda.synchronize()
    for r in got:
        for k in want:
            assert torch.equal(r[k], want[k]), k


def test_outputs_and_tensors_around_them_stay_as_they_were():
    """Buffers with guards on both sides: nothing outside the outputs and the workspace is written."""
    for G, S, M, V, dtype, K, piece in ((1, 37, 72, 301, "bf16", 3, 0), (1, 1500, 1024, 9001, "bf16", 0, 4096), (2, 33, 36, 101, "f32", 5, 0)):
        d = make(G, S, M, V, dtype, 0.3, K)
        sh, dims = moe.MoEShape(G, S, M, M, 2, 1, dtype), moe.VocabDims(V, K=K, temperature=2.0, piece=piece)
        guarded = []

        def guard(shape, dt):
            n = int(torch.tensor(shape).prod())
            pad = 4096 // torch.empty(0, dtype=dt).element_size()
            t = torch.full((n + 2 * pad,), 77, dtype=dt, device=DEV)
            guarded.append((t, pad, n))
            return t[pad:pad + n].view(shape)

        x, f32 = d["x"].view(G, S, M), torch.float32
        loss, lse = guard((G, S), f32), guard((G, S), f32)
        dx, dw = guard((G, S, M), x.dtype), guard((V, M), x.dtype)
        ws = guard((moe.moe_vocab_workspace_bytes(sh, dims),), torch.uint8)
        bws = guard((moe.moe_vocab_backward_workspace_bytes(sh, dims),), torch.uint8)
        dloss = d["dloss"].view(G, S)
        if K:
            entry, idx, logit = guard((G, S, K), f32), d["idx"].view(G, S, K), d["logit"].view(G, S, K)
            moe.moe_vocab_distill(sh, dims, x, d["w"], idx, logit, loss, lse, entry, ws)
            moe.moe_vocab_distill_backward(sh, dims, x, d["w"], idx, logit, entry, lse, dloss, dx, dw, bws)
        else:
            t = d["target"].view(G, S)
            moe.moe_vocab_loss(sh, dims, x, d["w"], t, loss, lse, ws)
            moe.moe_vocab_loss_backward(sh, dims, x, d["w"], t, loss, lse, dloss, dx, dw, bws)
        torch.cuda.synchronize()
        for t, pad, n in guarded:
            assert (t[:pad] == 77).all() and (t[pad + n:] == 77).all()
