"""The decoder's bridge to the encoder and the rest of a training step that tunes it.

  cross_forward    moe_cross_keys, moe_cross_attention   attention of a target's tokens to an encoder's states, from both sides' states
  cross_step       moe_cross_attention                   one step of generation: few tokens, keys and values in hand
  cross_backward   moe_cross_attention_backward          gradients of all inputs of cross_forward
  pref_forward     moe_preference_loss                   paired log ratios of whole sequences, from token losses
  pref_backward    moe_preference_loss_backward          their gradient at each token's loss
  policy_forward   moe_policy_loss                       clipped policy loss with a KL term, per token
  policy_backward  moe_policy_loss_backward              its gradient
  clip             moe_gradient_norm, moe_clip_gradients the norm over all gradients of some layers, and the clipped gradients

A case is a dict of plain values.  cross: B sources of up to Lk states, Lq target tokens each, model width M, ``heads`` of width d that
share ``kv_heads`` keys and values, ``ragged`` sources' lengths.  pref: P pairs of sequences of S tokens and fewer.  policy: G sequences
of S tokens.  clip: ``layers`` pairs of encoder layers' gradients.  The plain forms compute in 32 bits and round once; ``exact``
computes in 64.
"""
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _cross(name, op, B, Lq, Lk, M, heads, kv_heads, d, dtype="bf16", ragged=True):
    return {"name": name, "op": op, "B": B, "Lq": Lq, "Lk": Lk, "M": M, "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "ragged": ragged}


def _pref(name, op, P, S, kind="logistic", beta=0.1, smoothing=0.0):
    return {"name": name, "op": op, "P": P, "S": S, "kind": kind, "beta": beta, "smoothing": smoothing}


def _policy(name, op, G, S, low=0.2, high=0.2, beta=0.04, per_token=False):
    return {"name": name, "op": op, "G": G, "S": S, "low": low, "high": high, "beta": beta, "per_token": per_token}


def _clip(name, layers, M, H, A, E, dtype="bf16", ratio=0.5):
    return {"name": name, "op": "clip", "layers": layers, "M": M, "H": H, "A": A, "E": E, "dtype": dtype, "ratio": ratio}


def listed():
    return [
        # training of a paper-sized decoder layer: 32 sentence pairs of full length
        _cross("cross_forward_paper", "cross_forward", 32, 1024, 1024, 1024, 16, 16, 128, ragged=False),
        # the precision the paper trained in, a small batch whose source is longer than its target; nothing is round
        _cross("cross_forward_f32", "cross_forward", 5, 187, 411, 516, 8, 8, 64, "f32"),
        # the next token of one sentence, four hypotheses: the smallest call
        _cross("cross_step_sentence", "cross_step", 1, 4, 53, 1024, 16, 16, 128),
        # the next token of 64 documents: the keys and values are what is read
        _cross("cross_step_documents", "cross_step", 64, 1, 2048, 1024, 16, 16, 128),
        # the training step of the first case: the largest work here
        _cross("cross_backward_paper", "cross_backward", 32, 1024, 1024, 1024, 16, 16, 128, ragged=False),
        # sources of all lengths, four heads a key
        _cross("cross_backward_ragged", "cross_backward", 11, 333, 777, 776, 16, 4, 64),
        # 64 pairs of answers to prompts
        _pref("pref_forward", "pref_forward", 64, 2048),
        _pref("pref_backward", "pref_backward", 64, 2048, smoothing=0.1),
        # 512 sampled answers, advantages by answer
        _policy("policy_forward", "policy_forward", 512, 2048),
        # a minibatch of one device's tokens, advantages by token
        _policy("policy_backward", "policy_backward", 8, 4096, high=0.28, per_token=True),
        # what moe_encoder_pair_backward leaves at the paper's sizes
        _clip("clip_paper", 1, 1024, 8192, 2048, 32),
        # a deep small model in full precision: many tensors, some tiny
        _clip("clip_small_f32", 6, 128, 512, 128, 4, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["cross_forward", "cross_step", "cross_backward", "cross_forward", "cross_step", "cross_backward",
                     "pref_forward", "pref_backward", "policy_forward", "policy_backward", "clip"])
    if op.startswith("cross"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        unit = 8 if dtype == "bf16" else 4
        d = rng.choice([64, 128])
        share = rng.choice([1, 1, 1, 2, 4, 8])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        heads = min(kv_heads * share, 2048 // d)
        heads -= heads % kv_heads
        while (heads // kv_heads) & (heads // kv_heads - 1):
            heads -= kv_heads
        M = unit * _log(rng, 128 // unit, 1536 // unit)
        if op == "cross_step":
            B, Lq, Lk = _log(rng, 1, 64), rng.choice([1, 1, 2, 4, 5, 8, 16]), _log(rng, 1, 8192)
            Lk = max(1, min(Lk, (1 << 28) // (B * kv_heads * d * 4 * 2)))
        else:
            B, Lq, Lk = _log(rng, 1, 32), _log(rng, 1, 2048), _log(rng, 1, 2048)
            most = 2.5e11 if dtype == "bf16" else 2.0e10
            while B > 1 and 4.0 * B * Lq * Lk * heads * d + 4.0 * B * (Lq + Lk) * M * heads * d > most:
                B -= 1
        return _cross("", op, B, Lq, Lk, M, heads, kv_heads, d, dtype, rng.random() < 0.7)
    if op.startswith("pref"):
        return _pref("", op, _log(rng, 1, 256), _log(rng, 1, 4096), rng.choice(["logistic", "logistic", "squared"]),
                     round(0.05 + 0.45 * rng.random(), 3), rng.choice([0.0, 0.0, round(0.3 * rng.random(), 3)]))
    if op.startswith("policy"):
        return _policy("", op, _log(rng, 1, 512), _log(rng, 1, 4096), round(0.1 + 0.2 * rng.random(), 3),
                       round(0.1 + 0.3 * rng.random(), 3), rng.choice([0.0, round(0.1 * rng.random(), 4)]), rng.random() < 0.5)
    return _clip("", rng.choice([1, 1, 2, 4, 8]), 8 * _log(rng, 4, 128), 8 * _log(rng, 8, 256), 64 * rng.choice([1, 2, 5, 8, 12]),
                 rng.choice([2, 4, 7, 16]), rng.choice(["bf16", "bf16", "f32"]), rng.choice([0.1, 0.5, 0.9, 1.5]))


# ---- inputs

def _lengths(case, g):
    B, Lk = case["B"], case["Lk"]
    if not case["ragged"]:
        return torch.full((B,), Lk, dtype=torch.int32, device=DEV)
    n = (Lk * (0.2 + 0.8 * torch.rand(B, generator=g, device=DEV))).int().clamp_(min=1)
    n[0] = Lk
    return n


def _prepare_cross(case, g):
    B, Lq, Lk, M, d, dt = (case[k] for k in ("B", "Lq", "Lk", "M", "d", "dtype"))
    A, Akv, dt = case["heads"] * d, case["kv_heads"] * d, DTYPES[dt]
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    st = {"op": case["op"], "heads": case["heads"], "kv_heads": case["kv_heads"], "d": d, "u": rand(B, Lq, M).to(dt),
          "wq": (1.5 * rand(M, A) / M ** 0.5).to(dt), "wo": (rand(A, M) / A ** 0.5).to(dt)}
    wkv = (rand(M, 2 * Akv) / M ** 0.5).to(dt)
    st["len"] = _lengths(case, g) if case["ragged"] else None
    mem = rand(B, Lk, M).to(dt)
    kv = (mem.float().view(B * Lk, M) @ wkv.float()).to(dt).view(B, Lk, 2 * Akv)
    if case["op"] == "cross_step":
        st["kv"] = kv
    else:
        st.update(mem=mem, wkv=wkv)
    if case["op"] == "cross_backward":
        st.update(kv=kv, dout=(1e-3 * rand(B, Lq, M)).to(dt))
    if own:
        import paper_2006_16668_amd as moe
        sh = moe.MoEShape(B, Lq, M, M, 2, 1, case["dtype"])
        dims = moe.CrossDims(B, Lq, Lk, case["heads"], d, case["kv_heads"])
        bytes_ = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
        st.update(sh=sh, dims=dims, out=torch.empty_like(st["u"]))
        if case["op"] == "cross_backward":
            st["fwd"] = bytes_(moe.moe_cross_train_workspace_bytes(sh, dims))
            moe.moe_cross_attention_train(sh, dims, st["u"], kv, st["len"], st["wq"], st["wo"], st["out"], st["fwd"])
            st["grads"] = {k: torch.empty_like(st[n]) for k, n in (("du", "u"), ("dmem", "mem"), ("dwq", "wq"), ("dwkv", "wkv"), ("dwo", "wo"))}
            st["ws"] = bytes_(moe.moe_cross_backward_workspace_bytes(sh, dims))
        else:
            if case["op"] == "cross_forward":
                st["kv_out"] = torch.empty_like(kv)
            st["ws"] = bytes_(moe.moe_cross_workspace_bytes(sh, dims))
    return st


def _prepare_pref(case, g):
    P, S = case["P"], case["S"]
    uniform = lambda *s: torch.rand(*s, generator=g, device=DEV)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    # sequences lie one behind the other; their tokens begin with a prompt that has no target; some room is left at the end
    n = (S * (0.3 + 0.7 * uniform(2 * P))).long().clamp_(min=1)
    start = torch.zeros(2 * P + 1, dtype=torch.int32, device=DEV)
    start[1:] = torch.cumsum(n, 0)
    N = 2 * P * S
    at = torch.arange(N, device=DEV)
    seq = torch.searchsorted(start, at, right=True) - 1
    inside = at < start[-1]
    seq = seq.clamp(max=2 * P - 1)
    prompt = (at - start[seq]) < (0.3 * uniform(2 * P) * n)[seq].long()
    target = torch.where(inside & ~prompt, (uniform(N) * 32000).long(), -1).int()
    ref = 2.0 * rand(N).abs() + 0.01
    nll = (ref + 0.3 * rand(N) / max(1.0, S / 64) ** 0.5).clamp_(min=0.0)
    st = {"op": case["op"], "kind": case["kind"], "beta": case["beta"], "smoothing": case["smoothing"], "P": P, "V": 32000,
          "nll": nll.view(2 * P, S), "ref": ref.view(2 * P, S), "target": target.view(2 * P, S), "start": start}
    if case["op"] == "pref_backward":
        st["ratio"] = _plain_pref_forward(st)["ratio"]                       # as the forward pass has left it
        st["dloss"] = (0.5 + uniform(P)) / P
    if own:
        import paper_2006_16668_amd as moe
        st["sh"] = moe.MoEShape(2 * P, S, 8, 8, 2, 1, "f32")
        st["dims"] = moe.PreferenceDims(P, st["V"], case["beta"], case["smoothing"], case["kind"])
        if case["op"] == "pref_backward":
            st["dnll"] = torch.empty_like(st["nll"])
        else:
            st.update(loss=torch.empty(P, device=DEV), out_ratio=torch.empty(2 * P, device=DEV))
    return st


def _prepare_policy(case, g):
    G, S = case["G"], case["S"]
    uniform = lambda *s: torch.rand(*s, generator=g, device=DEV)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    old = 2.0 * rand(G, S).abs() + 0.01
    nll = (old + 0.2 * rand(G, S)).clamp_(min=0.0)
    ref = (old + 0.4 * rand(G, S)).clamp_(min=0.0)
    length = (S * (0.3 + 0.7 * uniform(G, 1))).long().clamp_(min=1)
    target = torch.where(torch.arange(S, device=DEV) < length, (uniform(G, S) * 32000).long(), -1).int()
    st = {"op": case["op"], "low": case["low"], "high": case["high"], "beta": case["beta"], "V": 32000, "nll": nll, "old": old,
          "ref": ref if case["beta"] else None, "adv": rand(G, S) if case["per_token"] else rand(G), "target": target}
    if case["op"] == "policy_backward":
        st["dloss"] = (0.5 + uniform(G, S)) / (G * S)
    if own:
        import paper_2006_16668_amd as moe
        st["sh"] = moe.MoEShape(G, S, 8, 8, 2, 1, "f32")
        st["dims"] = moe.PolicyDims(st["V"], case["low"], case["high"], case["beta"])
        if case["op"] == "policy_backward":
            st["dnll"] = torch.empty(G, S, device=DEV)
        else:
            st.update(loss=torch.empty(G, S, device=DEV), kl=torch.empty(G, S, device=DEV) if case["beta"] else None)
    return st


def _gradient_shapes(case):
    """The gradients of a pair of encoder layers, in the order of its weights: shape, whether always in 32 bits."""
    M, H, A, E = (case[k] for k in ("M", "H", "A", "E"))
    one = [((M,), True)] * 8 + [((M, 3 * A), False), ((A, M), False)] * 2 + [((M, H), False), ((H, M), False), ((M, E), True),
                                                                           ((E, M, H), False), ((E, H, M), False)]
    return one * case["layers"]


def _views(shapes, dtype):
    """Tensors that lie one behind the other in a buffer for each type, from whole 256 bytes on."""
    place, size = [], {torch.float32: 0, dtype: 0}
    for shape, full in shapes:
        t = torch.float32 if full else dtype
        n = 1
        for s in shape:
            n *= s
        place.append((t, size[t], n, shape))
        size[t] += (n + 127) // 128 * 128
    flat = {t: torch.zeros(n, dtype=t, device=DEV) for t, n in size.items()}
    return flat, [flat[t][at:at + n].view(shape) for t, at, n, shape in place]


def _flat(buffers):
    return {str(t).split(".")[1]: v for t, v in buffers.items()}


def _prepare_clip(case, g):
    shapes, dt = _gradient_shapes(case), DTYPES[case["dtype"]]
    flat, grads = _views(shapes, dt)
    for t in grads:
        t.normal_(0.0, 1e-3, generator=g)
    total = sum(float(t.float().pow(2).sum()) for t in flat.values()) ** 0.5
    out, clipped = _views(shapes, dt)
    st = {"op": "clip", "flat": flat, "grads": grads, "out": out, "clipped": clipped, "max_norm": case["ratio"] * total}
    if own:
        import paper_2006_16668_amd as moe
        st["list"] = moe.GradientList(grads, clipped)
        st["norm"] = torch.empty(1, device=DEV)
        st["ws"] = torch.empty(moe.moe_gradient_norm_workspace_bytes(st["list"]), dtype=torch.uint8, device=DEV)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["op"].split("_")[0]
    return {"cross": _prepare_cross, "pref": _prepare_pref, "policy": _prepare_policy, "clip": _prepare_clip}[kind](case, g)


# ---- plain forms, in 32 bits

def _heads(t, heads, d):
    return t.view(t.shape[0], t.shape[1], heads, d).transpose(1, 2).contiguous()


def _plain_core(st, kv):
    """q, k, v by heads, and the probabilities; k and v repeated for the heads that share them."""
    B, Lq, M = st["u"].shape
    heads, kv_heads, d = st["heads"], st["kv_heads"], st["d"]
    q = _heads((st["u"].float().view(B * Lq, M) @ st["wq"].float()).view(B, Lq, heads * d), heads, d)
    share = heads // kv_heads
    k = _heads(kv[..., :kv_heads * d], kv_heads, d).repeat_interleave(share, 1)
    v = _heads(kv[..., kv_heads * d:], kv_heads, d).repeat_interleave(share, 1)
    s = q @ k.transpose(2, 3) / d ** 0.5
    if st["len"] is not None:
        past = torch.arange(kv.shape[1], device=DEV)[None, :] >= st["len"][:, None]
        s.masked_fill_(past[:, None, None, :], -torch.inf)
    e = torch.exp(s - s.max(3, keepdim=True).values)
    return q, k, v, e / e.sum(3, keepdim=True)


def _plain_cross_forward(st):
    B, Lq, M = st["u"].shape
    dt = st["u"].dtype
    if "mem" in st:
        _, Lk, _ = st["mem"].shape
        kv = (st["mem"].float().view(B * Lk, M) @ st["wkv"].float()).view(B, Lk, -1)
    else:
        kv = st["kv"].float()
    _, _, v, p = _plain_core(st, kv)
    ctx = (p @ v).transpose(1, 2).reshape(B * Lq, -1)
    out = {"out": (ctx @ st["wo"].float()).to(dt).view(B, Lq, M)}
    if "mem" in st:
        out["kv"] = kv.to(dt)
    return out


def _plain_cross_backward(st):
    B, Lq, M = st["u"].shape
    Lk, heads, kv_heads, d, dt = st["kv"].shape[1], st["heads"], st["kv_heads"], st["d"], st["u"].dtype
    q, k, v, p = _plain_core(st, st["kv"].float())
    flat = lambda t: t.transpose(1, 2).reshape(t.shape[0] * t.shape[2], -1)
    dout = st["dout"].float().view(B * Lq, M)
    dwo = flat(p @ v).t() @ dout
    dctx = _heads((dout @ st["wo"].float().t()).view(B, Lq, heads * d), heads, d)
    dv = p.transpose(2, 3) @ dctx
    dp = dctx @ v.transpose(2, 3)
    ds = p * (dp - (dp * p).sum(3, keepdim=True)) / d ** 0.5
    dq = flat(ds @ k)
    dk = ds.transpose(2, 3) @ q
    shared = lambda t: flat(t.view(B, kv_heads, heads // kv_heads, Lk, d).sum(2))
    dkv = torch.cat([shared(dk), shared(dv)], 1)
    return {"du": (dq @ st["wq"].float().t()).to(dt).view(B, Lq, M), "dmem": (dkv @ st["wkv"].float().t()).to(dt).view(B, Lk, M),
            "dwq": (st["u"].float().view(B * Lq, M).t() @ dq).to(dt), "dwkv": (st["mem"].float().view(B * Lk, M).t() @ dkv).to(dt),
            "dwo": dwo.to(dt)}


def _log_sigmoid(x):
    return torch.clamp(x, max=0.0) - torch.log1p(torch.exp(-x.abs()))


def _sequences(st):
    """Each token's sequence, and whether it counts."""
    N, P = st["target"].numel(), st["P"]
    at = torch.arange(N, device=DEV)
    seq = (torch.searchsorted(st["start"], at, right=True) - 1)
    there = (seq >= 0) & (seq < 2 * P) & (st["target"].view(-1) >= 0)
    return seq.clamp(0, 2 * P - 1), there


def _plain_pref_forward(st):
    seq, there = _sequences(st)
    d = torch.where(there, st["ref"].view(-1) - st["nll"].view(-1), 0.0)
    ratio = torch.zeros(2 * st["P"], dtype=torch.float64, device=DEV).index_add_(0, seq, d.double())
    h = ratio[0::2] - ratio[1::2]
    if st["kind"] == "logistic":
        x = st["beta"] * h
        loss = -(1.0 - st["smoothing"]) * _log_sigmoid(x) - st["smoothing"] * _log_sigmoid(-x)
    else:
        loss = (h - 0.5 / st["beta"]) ** 2
    return {"loss": loss.float(), "ratio": ratio.float()}


def _plain_pref_backward(st):
    seq, there = _sequences(st)
    h = st["ratio"][0::2] - st["ratio"][1::2]
    if st["kind"] == "logistic":
        x = st["beta"] * h
        dh = st["beta"] * (st["smoothing"] / (1.0 + torch.exp(-x)) - (1.0 - st["smoothing"]) / (1.0 + torch.exp(x)))
    else:
        dh = 2.0 * h - 1.0 / st["beta"]
    dh = dh * st["dloss"]
    by_sequence = torch.stack([-dh, dh], 1).view(-1)
    return {"dnll": torch.where(there, by_sequence[seq], 0.0).view(st["nll"].shape)}


def _policy_ratio(st):
    """The advantages, the ratio, and where the bound stops it: ratios next to the bound are told apart in 64 bits."""
    adv = st["adv"] if st["adv"].dim() == 2 else st["adv"][:, None]
    r = torch.exp(st["old"].double() - st["nll"].double())
    stopped = ((adv > 0) & (r > 1.0 + st["high"])) | ((adv < 0) & (r < 1.0 - st["low"]))
    return adv, r.float(), stopped


def _plain_policy_forward(st):
    there = st["target"] >= 0
    adv, r, stopped = _policy_ratio(st)
    loss = -adv * torch.where(stopped, torch.clamp(r, 1.0 - st["low"], 1.0 + st["high"]), r)
    out = {}
    if st["ref"] is not None:
        x = st["nll"].double() - st["ref"].double()                      # (e^x - 1 - x of a small x has lost it in 32 bits)
        kl = (torch.exp(x) - 1.0 - x).float()
        loss = loss + st["beta"] * kl
        out["kl"] = torch.where(there, kl, 0.0)
    out["loss"] = torch.where(there, loss, 0.0)
    return out


def _plain_policy_backward(st):
    there = st["target"] >= 0
    adv, r, stopped = _policy_ratio(st)
    g = torch.where(stopped, 0.0, r * adv)
    if st["ref"] is not None:
        g = g + st["beta"] * (torch.exp(st["nll"].double() - st["ref"].double()) - 1.0).float()
    return {"dnll": torch.where(there, g * st["dloss"], 0.0)}


def _plain_clip(st):
    total = torch.zeros((), device=DEV)
    for t in st["grads"]:
        f = t.float()
        total = total + (f * f).sum()
    norm = torch.sqrt(total)
    scale = torch.clamp(st["max_norm"] / norm, max=1.0)
    for t, c in zip(st["grads"], st["clipped"]):
        c.copy_(t.float() * scale)
    return {"norm": norm.view(1), **_flat(st["out"])}


PLAIN = {"cross_forward": _plain_cross_forward, "cross_step": _plain_cross_forward, "cross_backward": _plain_cross_backward,
         "pref_forward": _plain_pref_forward, "pref_backward": _plain_pref_backward, "policy_forward": _plain_policy_forward,
         "policy_backward": _plain_policy_backward, "clip": _plain_clip}


# ---- the framework's calls

def _own(st):
    import paper_2006_16668_amd as moe
    op = st["op"]
    if op == "cross_forward":
        moe.moe_cross_keys(st["sh"], st["dims"], st["mem"], st["wkv"], st["kv_out"])
        moe.moe_cross_attention(st["sh"], st["dims"], st["u"], st["kv_out"], st["len"], st["wq"], st["wo"], st["out"], st["ws"])
        return {"out": st["out"], "kv": st["kv_out"]}
    if op == "cross_step":
        moe.moe_cross_attention(st["sh"], st["dims"], st["u"], st["kv"], st["len"], st["wq"], st["wo"], st["out"], st["ws"])
        return {"out": st["out"]}
    if op == "cross_backward":
        moe.moe_cross_attention_backward(st["sh"], st["dims"], st["u"], st["mem"], st["kv"], st["len"], st["wq"], st["wkv"], st["wo"],
                                         st["dout"], st["fwd"], st["grads"], st["ws"])
        return dict(st["grads"])
    if op == "pref_forward":
        moe.moe_preference_loss(st["sh"], st["dims"], st["nll"], st["ref"], st["target"], st["start"], st["loss"], st["out_ratio"])
        return {"loss": st["loss"], "ratio": st["out_ratio"]}
    if op == "pref_backward":
        moe.moe_preference_loss_backward(st["sh"], st["dims"], st["target"], st["start"], st["ratio"], st["dloss"], st["dnll"])
        return {"dnll": st["dnll"]}
    if op == "policy_forward":
        moe.moe_policy_loss(st["sh"], st["dims"], st["nll"], st["old"], st["ref"], st["adv"], st["target"], st["loss"], st["kl"])
        return {"loss": st["loss"]} if st["kl"] is None else {"kl": st["kl"], "loss": st["loss"]}
    if op == "policy_backward":
        moe.moe_policy_loss_backward(st["sh"], st["dims"], st["nll"], st["old"], st["ref"], st["adv"], st["target"], st["dloss"], st["dnll"])
        return {"dnll": st["dnll"]}
    moe.moe_gradient_norm(st["list"], st["norm"], st["ws"])
    moe.moe_clip_gradients(st["list"], st["norm"], st["max_norm"])
    return {"norm": st["norm"], **_flat(st["out"])}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ---- the definitions in 64 bits

def _exact_cross(case, st):
    B, Lq, Lk, M, d = (case[k] for k in ("B", "Lq", "Lk", "M", "d"))
    H, K, share = case["heads"], case["kv_heads"], case["heads"] // case["kv_heads"]
    u, wq, wo = st["u"].double(), st["wq"].double(), st["wo"].double()
    backward = case["op"] == "cross_backward"
    given = "kv" in st
    kv = st["kv"].double() if given else torch.matmul(st["mem"].double(), st["wkv"].double())
    n = [Lk] * B if st["len"] is None else st["len"].tolist()
    out = torch.zeros(B, Lq, M, dtype=torch.float64, device=DEV)
    if backward:
        mem, wkv, dout = st["mem"].double(), st["wkv"].double(), st["dout"].double()
        du, dmem = torch.zeros_like(u), torch.zeros_like(mem)
        dwq, dwkv, dwo = torch.zeros_like(wq), torch.zeros_like(wkv), torch.zeros_like(wo)
    for b in range(B):
        q = torch.mm(u[b], wq).view(Lq, K, share, d).permute(1, 2, 0, 3).reshape(K, share * Lq, d)
        k = kv[b, :n[b], :K * d].reshape(n[b], K, d).permute(1, 0, 2)
        v = kv[b, :n[b], K * d:].reshape(n[b], K, d).permute(1, 0, 2)
        p = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5, 2)
        back = lambda t: t.view(K, share, Lq, d).permute(2, 0, 1, 3).reshape(Lq, H * d)
        ctx = torch.bmm(p, v.contiguous())
        if not backward:
            out[b] = torch.mm(back(ctx), wo)
            continue
        dwo += torch.mm(back(ctx).t(), dout[b])
        dc = torch.mm(dout[b], wo.t()).view(Lq, K, share, d).permute(1, 2, 0, 3).reshape(K, share * Lq, d)
        ds = torch.bmm(dc, v.transpose(1, 2).contiguous())
        ds = (ds - (dc * ctx).sum(2, keepdim=True)) * p * d ** -0.5
        dq = back(torch.bmm(ds, k.contiguous()))
        dk = torch.bmm(ds.transpose(1, 2).contiguous(), q)
        dv = torch.bmm(p.transpose(1, 2).contiguous(), dc)
        dkv = torch.cat([t.permute(1, 0, 2).reshape(n[b], K * d) for t in (dk, dv)], 1)
        du[b] = torch.mm(dq, wq.t())
        dwq += torch.mm(u[b].t(), dq)
        dmem[b, :n[b]] = torch.mm(dkv, wkv.t())
        dwkv += torch.mm(mem[b, :n[b]].t(), dkv)
    if backward:
        return {"du": du, "dmem": dmem, "dwq": dwq, "dwkv": dwkv, "dwo": dwo}
    return {"out": out} if given else {"out": out, "kv": kv}


def _exact_pref(case, st):
    P, kind, beta, e = case["P"], case["kind"], case["beta"], case["smoothing"]
    edges = st["start"].tolist()
    counts = st["target"].view(-1) >= 0
    if case["op"] == "pref_forward":
        diff = ((st["ref"].double() - st["nll"].double()).view(-1) * counts).cpu()
        ratio = torch.tensor([float(diff[a:b].sum()) for a, b in zip(edges, edges[1:])], dtype=torch.float64, device=DEV)
        h = ratio.view(P, 2) @ torch.tensor([1.0, -1.0], dtype=torch.float64, device=DEV)
        if kind == "logistic":
            F = torch.nn.functional
            loss = (1 - e) * F.softplus(-beta * h, threshold=700) + e * F.softplus(beta * h, threshold=700)
        else:
            loss = torch.square(h - 1 / (2 * beta))
        return {"loss": loss, "ratio": ratio}
    r = st["ratio"].double().view(P, 2)
    h = r[:, 0] - r[:, 1]
    slope = beta * (torch.sigmoid(beta * h) - (1 - e)) if kind == "logistic" else 2 * (h - 1 / (2 * beta))
    slope = slope * st["dloss"].double()
    g = torch.zeros(counts.numel(), dtype=torch.float64, device=DEV)
    for i, (a, b) in enumerate(zip(edges, edges[1:])):
        g[a:b] = slope[i // 2] * (1 if i % 2 else -1)
    return {"dnll": (g * counts).view(st["nll"].shape)}


def _exact_policy(case, st):
    f = lambda k: st[k].double()
    a = f("adv") if case["per_token"] else f("adv").unsqueeze(1).expand(case["G"], case["S"])
    logr = f("old") - f("nll")
    r = logr.exp()
    lo, hi = 1 - case["low"], 1 + case["high"]
    stopped = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
    counts = st["target"] >= 0
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    x = f("nll") - f("ref") if st["ref"] is not None else None
    if case["op"] == "policy_backward":
        g = torch.where(stopped, zero, a * r)
        if x is not None:
            g = g + case["beta"] * x.expm1()
        return {"dnll": torch.where(counts, g * f("dloss"), zero)}
    bounded = torch.where(stopped, torch.where(a > 0, zero + hi, zero + lo), r)
    loss, out = -a * bounded, {}
    if x is not None:
        kl = x.expm1() - x
        loss = loss + case["beta"] * kl
        out["kl"] = torch.where(counts, kl, zero)
    out["loss"] = torch.where(counts, loss, zero)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["op"].split("_")[0]
    if kind != "clip":
        return {"cross": _exact_cross, "pref": _exact_pref, "policy": _exact_policy}[kind](case, st)
    norm = sum(float(torch.dot(t.double(), t.double())) for t in st["flat"].values()) ** 0.5
    scale = 1.0 if norm <= st["max_norm"] else st["max_norm"] / norm
    return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV), **{k: t.double() * scale for k, t in _flat(st["flat"]).items()}}


def work(case):
    """What a pass cannot do without: inputs and outputs once, and the products.  Ragged sources count by their mean length."""
    op = case["op"]
    if op.startswith("cross"):
        B, Lq, Lk, M, b = case["B"], case["Lq"], case["Lk"], case["M"], 4 if case["dtype"] == "f32" else 2
        A, Akv = case["heads"] * case["d"], case["kv_heads"] * case["d"]
        mean = (0.6 * Lk * (B - 1) + Lk) / B if case["ragged"] else Lk
        N, rows = B * Lq, B * Lk
        pairs = N * mean * A
        weights = 2 * M * A
        if op == "cross_step":
            return {"bytes": int((2 * N * M + weights + 2 * B * mean * Akv) * b), "flops": int(4 * N * M * A + 4 * pairs)}
        if op == "cross_forward":
            return {"bytes": (2 * N * M + rows * M + weights + 2 * M * Akv + 2 * rows * Akv) * b,
                    "flops": int(4 * N * M * A + 4 * rows * M * Akv + 4 * pairs)}
        return {"bytes": (3 * N * M + 2 * rows * M + 2 * (weights + 2 * M * Akv) + 2 * rows * Akv + 2 * N * A) * b,
                "flops": int(8 * N * M * A + 8 * rows * M * Akv + 10 * pairs)}
    if op.startswith("pref"):
        P, N = case["P"], 2 * case["P"] * case["S"]
        return {"bytes": (12 if op == "pref_forward" else 8) * N + 20 * P, "flops": (2 if op == "pref_forward" else 1) * N}
    if op.startswith("policy"):
        G, N = case["G"], case["G"] * case["S"]
        words = 3 + (1 if case["beta"] else 0) + (1 if case["per_token"] else 0)           # nll, old, target, ref, adv
        words += (1 + (1 if case["beta"] else 0)) if op == "policy_forward" else 2
        return {"bytes": 4 * N * words + (0 if case["per_token"] else 4 * G), "flops": 12 * N}
    size, count = 0, 0
    for shape, full in _gradient_shapes(case):
        n = 1
        for s in shape:
            n *= s
        count += n
        size += n * (4 if full or case["dtype"] == "f32" else 2)
    return {"bytes": 2 * size, "flops": 3 * count}
