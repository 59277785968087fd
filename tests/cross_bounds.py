"""Cross attention in 64 bits, and how far a call's results may be from it, element by element.

u = 2^-24 and h is the half step of the element type (bf16 2^-8, fp32 u).  A sum of n fp32 terms is off by at most n u of the sum of their magnitudes.
With scores s = q.k scale:

  scores         e_s = (d + 4) u (|q|.|k|) scale, and what q's own error leaves
  probabilities  p relative: e_p = 2 max e_s + (12 + max |s|) u   (an exponential of a difference with a rounded statistic; their sum's error is
                 one more e_p), and h for the rounding in front of a product
  ctx            (2 e_p + h + n u) sum p |v| + h |ctx|
  D              (h + (d + n) u + 2 e_p) |dctx|.(sum p |v|) + h |dctx|.|ctx|   (the stored ctx carries its own error)
  dS             p scale (e_dp + e_D) + (e_p + h + 3 u) p scale (|dctx|.|v| + |D|),   e_dp = d u |dctx|.|v|
  dq, dk, dv     the sums of these over states or queries, n u of the terms' magnitudes, and h of the result
"""
import torch

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def by_key_heads(t, kv_heads, share, d):
    """[B,L,kv_heads share d] -> [B,kv_heads,L share,d]: the columns of each key head."""
    B, L, _ = t.shape
    return t.view(B, L, kv_heads, share, d).permute(0, 2, 1, 3, 4).reshape(B, kv_heads, L * share, d)


def from_key_heads(t, L):
    B, K, C, d = t.shape
    return t.view(B, K, L, C // L, d).permute(0, 2, 1, 3, 4).reshape(B, L, K * (C // L) * d)


def core(q, kv, n, kv_heads, share, d, dtype, dctx=None, q_err=None):
    """q, dctx [B,Lq,A], kv [B,Lk,2 Akv] (any type), n: states that hold.  Values and bounds of ctx, and with dctx of dq, dkv."""
    h = HALF[dtype]
    B, Lq, _ = q.shape
    Lk = kv.shape[1]
    Akv = kv_heads * d
    holds = torch.arange(Lk, device=q.device)[None, :] < torch.as_tensor(n, device=q.device).view(B, 1)
    kv = torch.where(holds[:, :, None], kv.double(), 0.0)
    heads = lambda t: by_key_heads(t, kv_heads, share, d)
    flip = lambda t: t.transpose(2, 3).contiguous()
    Q = heads(q.double())
    K, V = (t.reshape(B, Lk, kv_heads, d).transpose(1, 2).contiguous() for t in (kv[..., :Akv], kv[..., Akv:]))
    scale = d ** -0.5
    mask = holds[:, None, None, :]
    s = torch.where(mask, Q @ flip(K) * scale, -torch.inf)
    m = s.max(3, keepdim=True).values
    m = torch.where(torch.isfinite(m), m, 0.0)
    p = torch.exp(s - m)
    total = p.sum(3, keepdim=True)
    p = torch.where(mask, p / torch.where(total > 0, total, 1.0), 0.0)
    e_s = (d + 4) * U * (Q.abs() @ flip(K.abs())) * scale
    if q_err is not None:
        e_s = e_s + heads(q_err) @ flip(K.abs()) * scale
    largest = torch.where(mask, s.abs(), 0.0).amax(3, keepdim=True)
    e_p = 2 * torch.where(mask, e_s, 0.0).amax(3, keepdim=True) + (12 + largest) * U
    terms = Lk
    ctx = p @ V
    pv = p @ V.abs()
    e_ctx = (2 * e_p + h + terms * U) * pv + h * ctx.abs()
    out = {"ctx": (from_key_heads(ctx, Lq), from_key_heads(e_ctx, Lq))}
    if dctx is None:
        return out
    G = heads(dctx.double())
    dp, dpa = G @ flip(V), G.abs() @ flip(V.abs())
    D = (G * ctx).sum(3, keepdim=True)
    e_D = ((G.abs() * (e_ctx + d * U * ctx.abs())).sum(3, keepdim=True))
    ds = p * (dp - D) * scale
    e_ds = p * scale * (d * U * dpa + e_D) + (e_p + h + 3 * U) * p * scale * (dpa + D.abs())
    sum_q = lambda t: t.view(B, kv_heads, -1, t.shape[3])
    dq, dk, dv = ds @ K, flip(ds) @ Q, flip(p) @ G
    cols = Q.shape[2]
    e_dq = e_ds @ K.abs() + terms * U * (ds.abs() @ K.abs()) + h * dq.abs()
    e_dk = flip(e_ds) @ Q.abs() + cols * U * (flip(ds.abs()) @ Q.abs()) + h * dk.abs()
    if q_err is not None:
        e_dk = e_dk + flip(ds.abs()) @ heads(q_err)
    e_dv = (flip(p * (e_p + h)) + cols * U * flip(p)) @ G.abs() + h * dv.abs()
    rows = lambda t: t.transpose(1, 2).reshape(B, Lk, Akv)
    out["dq"] = (from_key_heads(dq, Lq), from_key_heads(e_dq, Lq))
    out["dkv"] = (torch.cat([rows(dk), rows(dv)], 2), torch.cat([rows(e_dk), rows(e_dv)], 2))
    return out


def assert_within(got, want, err, what):
    bad = ~((got.double() - want).abs() <= err + 1e-30)
    if bad.any():
        i = bad.nonzero()[0].tolist()
        ratio = ((got.double() - want).abs() / (err + 1e-30)).nan_to_num(float("inf")).max()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {i}: {got[tuple(i)].item()} for "
                             f"{want[tuple(i)].item()}, bound {err[tuple(i)].item()}; at most {float(ratio)} of the bound")
