"""Attention under a rule in 64 bits, from its definition, with a bound for each result's error that counts the roundings of the
kernels: u is half a unit in the last place of the type that tensors are stored in, and in bf16 the probabilities and dS are
rounded to it as well; everything else is fp32 (e = 2^-24 an operation, n e over a sum of n terms)."""
import math

import torch

E32 = 2.0 ** -24


def reference(q, k, v, do=None, order="full", scale=None, cap=0.0, slopes=None, q_docs=None, k_docs=None, prefix=None, q0=0, few=False):
    """q [nb, Sq, H, dh] etc. of any type; returns {name: (value, bound)} in float64 for o, lse and, with do, dq, dk, dv.  few: the
    bound of calls of few pairs, where what a weight's rounding leaves out is rounded by itself (u u of the weight is lost) and delta
    does not go by the rounded o."""
    bf16 = q.dtype == torch.bfloat16
    u = 2.0 ** -8 if bf16 else E32
    nb, Sq, H, dh = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    G = H // Hkv
    scale = 1.0 / math.sqrt(dh) if scale is None else scale
    i = torch.arange(Sq).view(-1, 1) + q0
    j = torch.arange(Sk).view(1, -1)
    see = torch.ones(nb, Sq, Sk, dtype=torch.bool)
    if order == "causal":
        see &= j <= i
    if order == "prefix":
        see &= (j <= i) | (j < prefix.view(-1, 1, 1))
    if q_docs is not None:
        see &= (q_docs.view(nb, -1, 1) == k_docs.view(nb, 1, -1)) & (q_docs >= 0).view(nb, -1, 1)
    live_q = torch.ones(nb, Sq, dtype=torch.bool) if q_docs is None else q_docs >= 0
    live_k = torch.ones(nb, Sk, dtype=torch.bool) if k_docs is None else k_docs >= 0

    def wide(x, live):      # [nb, heads, rows, dh], padding rows as zeros
        return torch.where(live.view(*live.shape, 1, 1), x.detach().cpu().double(), 0.0).permute(0, 2, 1, 3)

    Q = wide(q, live_q)
    K, V = (wide(x, live_k).repeat_interleave(G, 1) for x in (k, v))
    t = scale * Q @ K.transpose(2, 3)
    # error of a score: the product's sum, and a few operations on the score; twice that (and the row's statistic) on p
    dt = (dh + 8) * E32 * scale * (Q.abs() @ K.abs().transpose(2, 3))
    bent = torch.tanh(t / cap) if cap else torch.zeros_like(t)
    s = cap * bent if cap else t
    ds_ = dt + 16 * E32 * (cap + s.abs())
    if slopes is not None:
        bias = slopes.double().view(1, H, 1, 1) * (i - j).abs()
        s = s - bias
        ds_ = ds_ + 4 * E32 * bias.abs()
    see = see.view(nb, 1, Sq, Sk).expand(nb, H, Sq, Sk)
    s = s.masked_fill(~see, -math.inf)
    empty = ~see.any(-1, keepdim=True) if Sk else torch.ones(nb, H, Sq, 1, dtype=torch.bool)
    lse = torch.where(empty, -math.inf, torch.logsumexp(s, -1, keepdim=True)) if Sk else torch.full((nb, H, Sq, 1), -math.inf, dtype=torch.float64)
    p = torch.exp(s - torch.where(empty, 0.0, lse)).masked_fill(~see, 0.0)
    off = torch.where(see, ds_, 0.0).amax(-1, keepdim=True) if Sk else torch.zeros_like(lse)    # of any score of the row
    fin = torch.where(empty, 0.0, lse)
    dp_rel = 2.1 * off + (Sk + 16) * E32 + 8 * E32 * fin.abs()          # relative error of a probability
    o = p @ V
    aV = p @ V.abs()
    up = (u * u if few else u) if bf16 else 0.0
    sum_err = (up + dp_rel + (Sk + 2) * E32) * aV * (1 + u)
    o_err = sum_err + u * o.abs()
    back = lambda x: x.permute(0, 2, 1, 3)   # noqa: E731
    out = {"o": (back(o), back(o_err)),
           "lse": (lse[..., 0], (off + (Sk + 16) * E32 + 8 * E32 * fin.abs())[..., 0])}
    if do is None:
        return out
    dO = wide(do, live_q)
    dP = dO @ V.transpose(2, 3)
    delta = (p * dP).sum(-1, keepdim=True)
    delta_err = (dO.abs() * (sum_err + u ** 3 * o.abs() if few else o_err)).sum(-1, keepdim=True) + dh * E32 * (dO.abs() * o.abs()).sum(-1, keepdim=True)
    dP_err = (dh + 2) * E32 * (dO.abs() @ V.abs().transpose(2, 3))
    slope = 1.0 - bent * bent
    dS = p * (dP - delta) * slope
    dS_err = (up + dp_rel + 16 * E32) * dS.abs() + p * (dP_err + delta_err) * (1 + dp_rel) + p * (dP - delta).abs() * (8 * E32 + (2 * dt / cap if cap else 0.0))
    # a query whose p is within 2^-16 (bf16) or 2^-18 of 1 is taken to see one key, dS = 0
    dS_err = dS_err + torch.where(p > 1 - (2.0 ** -15 if bf16 else 2.0 ** -17), dS.abs(), 0.0)
    dv = p.transpose(2, 3) @ dO
    dv_err = p.transpose(2, 3) @ ((up + dp_rel + (G * Sq + 4) * E32) * dO.abs()) * (1 + u)
    dq = scale * dS @ K
    dq_err = scale * (dS_err + (Sk + 4) * E32 * dS.abs()) @ K.abs() * (1 + u) + u * dq.abs()
    dk = scale * dS.transpose(2, 3) @ Q
    dk_err = scale * (dS_err + (G * Sq + 4) * E32 * dS.abs()).transpose(2, 3) @ Q.abs() * (1 + u)
    share = lambda x: x.view(nb, Hkv, G, Sk, dh).sum(2)   # noqa: E731
    dk, dk_err, dv, dv_err = (share(x) for x in (dk, dk_err, dv, dv_err))
    out["dq"] = back(dq), back(dq_err)
    out["dk"] = back(dk), back(dk_err + u * dk.abs())
    out["dv"] = back(dv), back(dv_err + u * dv.abs())
    return out


def check(name, got, want):
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    inf = torch.isinf(value)
    assert torch.equal(got[inf], value[inf]), name
    assert torch.isfinite(got[~inf]).all(), f"{name}: not finite"
    bad = (got - value).abs()[~inf] - (bound[~inf] + 1e-30)
    assert bad.numel() == 0 or float(bad.max()) <= 0, f"{name}: {float((got - value).abs()[~inf].max())} off, {int((bad > 0).sum())} values beyond their bound"
