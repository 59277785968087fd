"""The end of a model in training: what turns the last hidden states into a loss and brings its gradient back.

  ce_forward   moe_vocab_loss               softmax cross entropy over a vocabulary, x [N,M] and w [V,M] in, logits never kept
  ce_backward  moe_vocab_loss_backward      its gradients dx [N,M] and dw [V,M]
  kd_forward   moe_vocab_distill            cross entropy against the softmax of a teacher's K largest logits, minus its entropy
  kd_backward  moe_vocab_distill_backward   its gradients
  ln_forward   moe_add_layer_norm           s = x + delta, n = LN(s), rows of any width
  ln_backward  moe_add_layer_norm_backward  ds, dgamma and dbeta of it

A case is a dict of plain values: ``op`` as above, G groups of S tokens (N = G S), width M, vocabulary V, K teacher entries,
the temperature T of a distillation, ``empty`` the share of tokens without a target (padding, prompts), ``dtype``.  The plain
forms compute in 32 bits and round once; ``exact`` computes in 64.
"""
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _vocab(name, op, G, S, M, V, dtype="bf16", empty=0.0, K=0, T=1.0):
    return {"name": name, "op": op, "G": G, "S": S, "M": M, "V": V, "dtype": dtype, "empty": empty, "K": K, "T": T}


def _norm(name, op, G, S, M, dtype="bf16", residual=True):
    return {"name": name, "op": op, "G": G, "S": S, "M": M, "dtype": dtype, "residual": residual}


def listed():
    return [
        # the loss of one device's share of tokens, paper-sized width, the 32k vocabulary of its one-language models; a few
        # positions are padding
        _vocab("ce_forward_paper", "ce_forward", 8, 4096, 1024, 32000, empty=0.05),
        # scoring one token: all of the vocabulary's weights for one row
        _vocab("ce_forward_token", "ce_forward", 1, 1, 1024, 32000),
        # the training step of the first case: the largest work here
        _vocab("ce_backward_paper", "ce_backward", 8, 4096, 1024, 32000, empty=0.05),
        # three sequences of an instruction data set: most positions are prompt and have no target; nothing is round
        _vocab("ce_backward_prompts", "ce_backward", 3, 1021, 776, 50257, empty=0.6),
        # the precision the paper trained in
        _vocab("ce_backward_f32", "ce_backward", 2, 750, 512, 16001, "f32", empty=0.1),
        # a student of the 64k vocabulary that learns from the 32 largest logits its teacher stored per token
        _vocab("kd_forward", "kd_forward", 4, 2048, 1024, 64000, empty=0.02, K=32, T=2.0),
        _vocab("kd_backward", "kd_backward", 4, 2048, 1024, 64000, empty=0.02, K=32, T=2.0),
        # a microbatch of two dozen tokens
        _vocab("kd_backward_few", "kd_backward", 1, 24, 1024, 32000, K=8, T=1.0),
        # rows wider than a wavefront holds in registers, in full precision
        _norm("ln_forward_wide_f32", "ln_forward", 2, 1500, 5120, "f32"),
        # the norm in front of the loss of the first case, with the residual branch's gradient
        _norm("ln_backward_paper", "ln_backward", 8, 4096, 1024),
        # the smallest call: launches and latency only
        _norm("ln_backward_small_f32", "ln_backward", 1, 37, 520, "f32", residual=False),
        # a wide model's rows
        _norm("ln_backward_wide", "ln_backward", 2, 2048, 8192),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["ce_forward", "ce_backward", "kd_forward", "kd_backward", "ln_forward", "ln_backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    unit = 8 if dtype == "bf16" else 4
    G = rng.choice([1, 1, 2, 3, 8])
    if op.startswith("ln"):
        M = unit * _log(rng, 64 // unit, 16384 // unit)
        S = _log(rng, 1, max(1, min(32768, (1 << 25) // M) // G))
        return _norm(None, op, G, S, M, dtype, rng.random() < 0.5) | {"name": ""}
    M = unit * _log(rng, 64 // unit, 2048 // unit)
    V = _log(rng, 200, 131072)
    most = (1.0e12 if dtype == "bf16" else 6.0e10) / (M * V)
    S = _log(rng, 1, max(1, int(min(32768, most) / G)))
    K = _log(rng, 1, min(64, V // 2)) if op.startswith("kd") else 0
    T = round(1.0 + 3.0 * rng.random(), 2) if K else 1.0
    return _vocab("", op, G, S, M, V, dtype, round(0.8 * rng.random() ** 2, 3), K, T)


def _filled(case):
    """How many tokens have a target."""
    N = case["G"] * case["S"]
    return N - int(case["empty"] * N)


def _shape(case):
    import paper_2006_16668_amd as moe
    return moe.MoEShape(case["G"], case["S"], case["M"], case["M"], 2, 1, case["dtype"])


def _prepare_norm(case, g):
    N, M, dt = case["G"] * case["S"], case["M"], DTYPES[case["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    st = {"op": case["op"], "gamma": 1.0 + 0.1 * rand(M), "beta": 0.1 * rand(M)}
    dims = (case["G"], case["S"], M)
    x = (rand(N, M) * (0.5 + 2.0 * torch.rand(N, 1, generator=g, device=DEV)) + 0.3 * rand(N, 1)).to(dt).view(dims)
    extra = (0.5 * rand(N, M)).to(dt).view(dims) if case["residual"] else None
    if case["op"] == "ln_forward":
        st.update(x=x, delta=extra)
    else:
        st.update(s=x, dn=(1e-3 * rand(N, M)).to(dt).view(dims), dres=None if extra is None else (2e-3 * extra).to(dt))
    if own:
        import paper_2006_16668_amd as moe
        sh = _shape(case)
        st["sh"] = sh
        if case["op"] == "ln_forward":
            st.update(sum_out=torch.empty_like(x) if extra is not None else None, norm_out=torch.empty_like(x))
        else:
            st.update(ds=torch.empty_like(x), dgamma=torch.empty(M, device=DEV), dbeta=torch.empty(M, device=DEV),
                      ws=torch.empty(moe.moe_layer_norm_backward_workspace_bytes(sh), dtype=torch.uint8, device=DEV))
    return st


def _prepare_vocab(case, g):
    N, M, V, K, T, dt = case["G"] * case["S"], case["M"], case["V"], case["K"], case["T"], DTYPES[case["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    uniform = lambda *s: torch.rand(*s, generator=g, device=DEV)
    w = rand(V, M).mul_(2.0 / M ** 0.5).to(dt)
    filled = _filled(case)
    has = torch.zeros(N, dtype=torch.bool, device=DEV)
    has[torch.randperm(N, generator=g, device=DEV)[:filled]] = True
    st = {"op": case["op"], "w": w, "T": T}
    # words are used unevenly: low indices most; a token's hidden state leans towards what follows it, sure or not
    if K:
        idx = (torch.sort(uniform(N, K)).values ** 3 * (V - K)).long().clamp_(max=V - K) + torch.arange(K, device=DEV)
        idx = torch.gather(idx, 1, torch.argsort(uniform(N, K), dim=1))
        logit = torch.sort(2.0 * rand(N, K), dim=1, descending=True).values.contiguous()
        first = idx[:, 0]
        # stored lists are not all full
        short = (uniform(N, 1) < 0.1) & (torch.arange(K, device=DEV) >= (K + 1) // 2)
        idx = torch.where(has[:, None] & ~short, idx, -1)
        st.update(idx=idx.int().view(case["G"], case["S"], K), tlogit=logit.view(case["G"], case["S"], K))
    else:
        first = (uniform(N) ** 3 * V).long().clamp_(max=V - 1)
        st["target"] = torch.where(has, first, -1).int().view(case["G"], case["S"])
    x = rand(N, M) + 3.0 * uniform(N, 1) * w[first].float()
    st["x"] = x.to(dt).view(case["G"], case["S"], M)
    if case["op"].endswith("backward"):
        st["dloss"] = ((0.5 + uniform(N)) / max(filled, 1)).view(case["G"], case["S"])
        fwd = _plain_kd_forward(st) if K else _plain_ce_forward(st)          # what the forward pass has left
        st.update(fwd)
    if own:
        import paper_2006_16668_amd as moe
        sh, dims = _shape(case), moe.VocabDims(V, K=K, temperature=T)
        st.update(sh=sh, dims=dims)
        if case["op"].endswith("backward"):
            st.update(dx=torch.empty_like(st["x"]), dw=torch.empty_like(w))
            need = moe.moe_vocab_backward_workspace_bytes(sh, dims)
        else:
            out = lambda *s: torch.empty(case["G"], case["S"], *s, device=DEV)
            st.update(loss=out(), lse=out(), entry_logit=out(K) if K else None)
            need = moe.moe_vocab_workspace_bytes(sh, dims)
        st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return _prepare_norm(case, g) if case["op"].startswith("ln") else _prepare_vocab(case, g)


# ---- plain forms, in 32 bits

def _rows(st, key):
    """The rows with a target, and their x in 32 bits."""
    v = st[key].view(-1) >= 0 if key == "target" else (st[key] >= 0).any(-1).view(-1)
    rows = torch.nonzero(v).view(-1)
    M = st["x"].shape[-1]
    return rows, st["x"].view(-1, M)[rows].float()


def _log_sum_exp(z):
    m = z.max(1, keepdim=True).values
    return m.squeeze(1) + torch.log(torch.exp(z - m).sum(1))


def _teacher(st, rows, dtype=torch.float32):
    """Indices (0 for an absent entry), which are there, and the teacher's probabilities over them."""
    K = st["idx"].shape[-1]
    idx = st["idx"].view(-1, K)[rows].long()
    there = idx >= 0
    t = torch.where(there, st["tlogit"].view(-1, K)[rows].to(dtype), -torch.inf)
    q = torch.exp((t - t.max(1, keepdim=True).values) / st["T"])
    return idx.clamp(min=0), there, q / q.sum(1, keepdim=True)


def _spread(st, rows, values, *tail):
    shape = st["x"].shape[:2]
    out = torch.zeros(shape[0] * shape[1], *tail, dtype=values.dtype, device=DEV)
    out[rows] = values
    return out.view(*shape, *tail)


def _plain_ce_forward(st):
    rows, x = _rows(st, "target")
    z = x @ st["w"].float().t()
    lse = _log_sum_exp(z)
    zy = torch.gather(z, 1, st["target"].view(-1)[rows].long()[:, None]).squeeze(1)
    return {"loss": _spread(st, rows, lse - zy), "lse": _spread(st, rows, lse)}


def _plain_kd_forward(st):
    rows, x = _rows(st, "idx")
    z = x @ st["w"].float().t()
    idx, there, q = _teacher(st, rows)
    ze = torch.where(there, torch.gather(z, 1, idx), 0.0)
    lse = _log_sum_exp(z.div_(st["T"]))
    terms = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-45)) - ze / st["T"] + lse[:, None]), 0.0)
    return {"loss": _spread(st, rows, terms.sum(1)), "lse": _spread(st, rows, lse),
            "entry_logit": _spread(st, rows, ze, ze.shape[1])}


def _plain_backward(st):
    key = "idx" if "idx" in st else "target"
    rows, x = _rows(st, key)
    w = st["w"].float()
    g = st["dloss"].view(-1)[rows, None] / st["T"]
    d = x @ w.t()
    d = torch.exp_(d.div_(st["T"]).sub_(st["lse"].view(-1)[rows, None]))
    if key == "idx":
        idx, there, q = _teacher(st, rows)
        d.scatter_add_(1, idx, torch.where(there, -q, 0.0))
    else:
        d.scatter_add_(1, st["target"].view(-1)[rows].long()[:, None], -torch.ones_like(g))
    d.mul_(g)
    dt = st["x"].dtype
    return {"dx": _spread(st, rows, (d @ w).to(dt), x.shape[1]), "dw": (d.t() @ x).to(dt)}


def _plain_ln_forward(st):
    s = st["x"].float()
    if st["delta"] is not None:
        s = (s + st["delta"].float()).to(st["x"].dtype)
    v = s.float()
    c = v - v.mean(-1, keepdim=True)
    n = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6) * st["gamma"] + st["beta"]
    out = {"norm_out": n.to(st["x"].dtype)}
    if st["delta"] is not None:
        out["sum_out"] = s
    return out


def _plain_ln_backward(st):
    M = st["s"].shape[-1]
    v, dn = st["s"].float(), st["dn"].float()
    c = v - v.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6)
    xh = c * rstd
    g = dn * st["gamma"]
    ds = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    if st["dres"] is not None:
        ds = ds + st["dres"].float()
    return {"ds": ds.to(st["s"].dtype), "dgamma": (dn * xh).view(-1, M).sum(0), "dbeta": dn.view(-1, M).sum(0)}


PLAIN = {"ce_forward": _plain_ce_forward, "kd_forward": _plain_kd_forward, "ce_backward": _plain_backward,
         "kd_backward": _plain_backward, "ln_forward": _plain_ln_forward, "ln_backward": _plain_ln_backward}


# ---- the framework's calls

def _own(st):
    import paper_2006_16668_amd as moe
    op, sh = st["op"], st["sh"]
    if op == "ln_forward":
        moe.moe_add_layer_norm(sh, st["x"], st["delta"], st["gamma"], st["beta"], st["sum_out"], st["norm_out"])
        out = {"norm_out": st["norm_out"]}
        if st["delta"] is not None:
            out["sum_out"] = st["sum_out"]
        return out
    if op == "ln_backward":
        moe.moe_add_layer_norm_backward(sh, st["s"], st["dn"], st["gamma"], st["dres"], st["ds"], st["dgamma"], st["dbeta"],
                                        st["ws"])
        return {"ds": st["ds"], "dgamma": st["dgamma"], "dbeta": st["dbeta"]}
    if op == "ce_forward":
        moe.moe_vocab_loss(sh, st["dims"], st["x"], st["w"], st["target"], st["loss"], st["lse"], st["ws"])
        return {"loss": st["loss"], "lse": st["lse"]}
    if op == "kd_forward":
        moe.moe_vocab_distill(sh, st["dims"], st["x"], st["w"], st["idx"], st["tlogit"], st["loss"], st["lse"],
                              st["entry_logit"], st["ws"])
        return {"loss": st["loss"], "lse": st["lse"], "entry_logit": st["entry_logit"]}
    if op == "ce_backward":
        moe.moe_vocab_loss_backward(sh, st["dims"], st["x"], st["w"], st["target"], st["loss"], st["lse"], st["dloss"],
                                    st["dx"], st["dw"], st["ws"])
    else:
        moe.moe_vocab_distill_backward(sh, st["dims"], st["x"], st["w"], st["idx"], st["tlogit"], st["entry_logit"],
                                       st["lse"], st["dloss"], st["dx"], st["dw"], st["ws"])
    return {"dx": st["dx"], "dw": st["dw"]}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ---- the definitions in 64 bits

def _exact_norm(case, st):
    M = case["M"]
    if case["op"] == "ln_forward":
        s = st["x"].double()
        if st["delta"] is not None:
            s = (s + st["delta"].double())
            rounded = s.to(st["x"].dtype).double()               # what is normalised is the sum as it is stored
        else:
            rounded = s
        var, mean = torch.var_mean(rounded, -1, correction=0, keepdim=True)
        out = {"norm_out": (rounded - mean) * (var + 1e-6).rsqrt() * st["gamma"].double() + st["beta"].double()}
        if st["delta"] is not None:
            out["sum_out"] = s
        return out
    s, dn, gamma = (st[k].double() for k in ("s", "dn", "gamma"))
    var, mean = torch.var_mean(s, -1, correction=0, keepdim=True)
    r = (var + 1e-6).rsqrt()
    hat = (s - mean) * r
    up = dn * gamma
    ds = (up - (up.sum(-1, keepdim=True) + hat * (up * hat).sum(-1, keepdim=True)) / M) * r
    if st["dres"] is not None:
        ds += st["dres"].double()
    return {"ds": ds, "dgamma": (dn * hat).sum((0, 1)), "dbeta": dn.sum((0, 1))}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"].startswith("ln"):
        return _exact_norm(case, st)
    N, M, V, K, T = case["G"] * case["S"], case["M"], case["V"], case["K"], case["T"]
    w, x = st["w"].double(), st["x"].view(N, M)
    entries = st["idx"].view(N, K).long() if K else st["target"].view(N, 1).long()
    mass = st["tlogit"].view(N, K).double() if K else torch.zeros(N, 1, dtype=torch.float64, device=DEV)
    backward = case["op"].endswith("backward")
    new = lambda *s: torch.zeros(*s, dtype=torch.float64, device=DEV)
    loss, lse, ent = new(N), new(N), new(N, max(K, 1))
    dx, dw = (new(N, M), new(V, M)) if backward else (None, None)
    step = max(1, min(N, (1 << 28) // V))
    for a in range(0, N, step):
        e = entries[a:a + step]
        keep = (e >= 0).any(1).nonzero().view(-1) + a
        if keep.numel() == 0:
            continue
        e = entries[keep]
        absent = e < 0
        xr = x[keep].double()
        z = xr @ w.t() / T
        q = torch.softmax((mass[keep] / T).masked_fill(absent, -torch.inf), 1)
        ze = torch.gather(z, 1, e.clamp(min=0))
        l = torch.logsumexp(z, 1)
        if not backward:
            lse[keep] = l
            ent[keep] = (ze * T).masked_fill(absent, 0.0)
            loss[keep] = (torch.special.xlogy(q, q) - q * (ze - l[:, None])).sum(1)
            continue
        # the backward pass is a function of the statistics that it is given
        p = torch.exp(z - st["lse"].view(-1)[keep].double()[:, None])
        p.scatter_add_(1, e.clamp(min=0), -q)
        p *= st["dloss"].view(-1)[keep].double()[:, None] / T
        dx[keep] = p @ w
        dw += p.t() @ xr
    if backward:
        return {"dx": dx.view(st["x"].shape), "dw": dw}
    out = {"loss": loss.view(case["G"], case["S"]), "lse": lse.view(case["G"], case["S"])}
    if K:
        out["entry_logit"] = ent.view(case["G"], case["S"], K)
    return out


def work(case):
    """What a pass cannot do without: inputs and outputs once; one product of the filled rows with the vocabulary forward, three
    backward (the logits again, dx, dw)."""
    N, M, b = case["G"] * case["S"], case["M"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "ln_forward":
        return {"bytes": N * M * b * (4 if case["residual"] else 2) + 8 * M, "flops": 8 * N * M}
    if case["op"] == "ln_backward":
        return {"bytes": N * M * b * (4 if case["residual"] else 3) + 12 * M, "flops": 16 * N * M}
    V, K, n = case["V"], case["K"], _filled(case)
    if case["op"].endswith("forward"):
        return {"bytes": (n + V) * M * b + N * (8 + (12 * K if K else 4)), "flops": 2 * n * M * V}
    return {"bytes": (n + N + 2 * V) * M * b + N * (12 + (12 * K if K else 4)), "flops": 6 * n * M * V}
