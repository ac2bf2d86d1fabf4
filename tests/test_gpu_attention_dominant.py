"""Attention under a rule where one key takes nearly all of a query's weight, or is the only one that it sees: gradients relative to their
own size, and exact zeros.

Of such a row the dominant key m has dS_m = -(sum of the others' dS): as large as all of them together, and far smaller than what is left
of dP_m - delta if the two are rounded apart."""
import math

import pytest
import torch

from paper_2102_03161_amd import binding
from tests.test_gpu_attention_rules import compare

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24


def dominated(nb, S, H, dh, dtype, gaps, alone, gen):
    """q, k, v, dO and documents: one key of each query lies `gaps` above the logarithm of the sum of the others' weights.  alone: two
    keys a document, else all keys in one."""
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)   # noqa: E731
    k, v, do = ((x).to(dtype).double() for x in (r(nb, H, S, dh), r(nb, H, S, dh), r(nb, H, S, dh)))
    docs = (torch.arange(S) // 2 if alone else torch.zeros(S)).int().view(1, S).expand(nb, S).contiguous()
    see = docs.view(nb, 1, S, 1) == docs.view(nb, 1, 1, S)
    m = (torch.arange(S) ^ torch.randint(0, 2, (S,), generator=gen)) if alone else torch.randperm(S, generator=gen)
    way = k[:, :, m] - (k[:, :, m ^ 1] if alone else 0.0)
    want = gaps[0] + (gaps[1] - gaps[0]) * torch.rand(nb, H, S, 1, generator=gen, dtype=torch.float64)
    lo, hi = torch.zeros_like(want), torch.full_like(want, 64.0)
    own = torch.zeros(S, S, dtype=torch.bool)
    own[torch.arange(S), m] = True
    for _ in range(50):
        mid = (lo + hi) / 2
        s = (mid * way) @ k.transpose(2, 3) / math.sqrt(dh)
        gap = (s * own).sum(-1, keepdim=True) - torch.logsumexp(s.masked_fill(~see | own, -math.inf), -1, keepdim=True)
        lo, hi = torch.where(gap < want, mid, lo), torch.where(gap < want, hi, mid)
    back = lambda x: x.permute(0, 2, 1, 3).to(dtype)   # noqa: E731
    return back(hi * way), back(k), back(v), back(do), docs


def exact(q, k, v, do, docs, cap):
    """{name: (value, bound)}: see the comments."""
    bf16 = q.dtype == BF16
    u = 2.0 ** -8 if bf16 else E
    nb, S, H, dh = q.shape
    Q, K, V, dO = (x.double().permute(0, 2, 1, 3) for x in (q, k, v, do))
    scale = 1.0 / math.sqrt(dh)
    see = docs.view(nb, 1, S, 1) == docs.view(nb, 1, 1, S)
    t = scale * Q @ K.transpose(2, 3)
    bent = torch.tanh(t / cap) if cap else torch.zeros_like(t)
    s = (cap * bent if cap else t).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = torch.exp(s - lse)
    # a score: the product's sum in fp32 and some operations on it; a weight twice that, and what its row's statistic is off
    ds = (dh + 8) * E * scale * (Q.abs() @ K.abs().transpose(2, 3)) + 16 * E * (cap + torch.where(see, s, 0.0).abs())
    rel = 2.1 * torch.where(see, ds, 0.0).amax(-1, keepdim=True) + (S + 16) * E + 8 * E * lse.abs()
    dP = dO @ V.transpose(2, 3)
    mass = dO.abs() @ V.abs().transpose(2, 3)          # sum of |dO||v|: what the rounding of a dP counts against
    slope = 1.0 - bent * bent
    raw = p * (dP - (p * dP).sum(-1, keepdim=True))
    dS = raw * slope
    top = torch.zeros_like(see.expand_as(p)).scatter(-1, p.argmax(-1, keepdim=True), True)
    assert bool((p.amax(-1) > 0.9).all())
    mass_m = (mass * top).sum(-1, keepdim=True)
    # the others: their weight, and dP - delta, two fp32 sums over the head size (bf16: a weight is rounded, and so is its part in the
    # correction that takes out how far dO . o of the rounded o is from delta, 2^-8 of the mass)
    slope_err = 2.0 * ds / cap if cap else 0.0
    err = (rel + 16 * E + slope_err) * raw.abs() + p * (2 * dh + 4) * E * (mass + mass_m)
    if bf16:
        err = err + u * raw.abs() + 2 * u * p * ((dP - (p * dP).sum(-1, keepdim=True)).abs() + u * mass_m)
    err = torch.where(see & ~top, err, 0.0)
    others = err.sum(-1, keepdim=True)
    # the dominant one: minus their sum.  bf16, keys' and values' gradients: p (dP - delta) of one delta in fp32, off by half a unit
    # of delta and of the two sums that it is made of, the products being the same
    err_k = err + torch.where(top, others + (slope_err + 16 * E) * raw.abs() + (u * raw.abs() + 8 * E * mass if bf16 else 0.0), 0.0)
    # bf16, queries' gradients: as above; under a cap the weight in the correction is not 1 but a slope, rounded
    err_q = err + torch.where(top, others + (slope_err + 16 * E) * raw.abs() + ((2 * u * u * mass if cap else 8 * E * mass) if bf16 else 0.0), 0.0)
    dq, dk = scale * dS @ K, scale * dS.transpose(2, 3) @ Q
    n = (S + 4) * E
    dq_err = scale * (err_q * slope + n * dS.abs()) @ K.abs() * (1 + u) + u * dq.abs()
    dk_err = scale * (err_k * slope + n * dS.abs()).transpose(2, 3) @ Q.abs() * (1 + u) + u * dk.abs()
    back = lambda x: x.permute(0, 2, 1, 3)   # noqa: E731
    return dict(dq=(back(dq), back(dq_err)), dk=(back(dk), back(dk_err)))


def gradients(q, k, v, do, docs, cap=0.0):
    q, k, v, do = (x.cuda() for x in (q, k, v, do))
    rule = binding.AttentionRule(cap=cap, documents=docs.cuda())
    o, lse = binding.attention_forward(q, k, v, rule)
    dq, dk, dv = binding.attention_backward(q, k, v, o, lse, do, rule)
    return dict(o=o.cpu(), dq=dq.cpu(), dk=dk.cpu(), dv=dv.cpu())


def check(q, k, v, do, docs, cap):
    want, got = exact(q, k, v, do, docs, cap), gradients(q, k, v, do, docs, cap)
    for name, (value, bound) in want.items():
        off = (got[name].double() - value).abs()
        size = value.abs().mean()
        print(f"  {name}: off {float(off.mean() / size):.2e} of its size, bound {float(bound.mean() / size):.2e}", flush=True)
        assert (off <= bound).all(), (name, float((off / bound).max()))


@pytest.mark.parametrize("alone", [True, False], ids=["two keys", "all keys"])
@pytest.mark.parametrize("nb,S,H,dh,cap", [(1, 64, 2, 64, 0.0), (2, 130, 3, 64, 0.0), (1, 70, 2, 128, 0.0), (6, 320, 16, 64, 0.0), (1, 130, 2, 32, 60.0)])
def test_dominant_keys_in_fp32(nb, S, H, dh, cap, alone):
    gen = torch.Generator().manual_seed(S + dh)
    check(*dominated(nb, S, H, dh, F32, (13.0, 16.0), alone, gen), cap)


@pytest.mark.parametrize("alone", [True, False], ids=["two keys", "all keys"])
@pytest.mark.parametrize("nb,S,H,dh", [(1, 64, 2, 64), (2, 130, 3, 64), (1, 70, 2, 128), (22, 260, 8, 64)])
def test_dominant_keys_in_bf16(nb, S, H, dh, alone):
    gen = torch.Generator().manual_seed(S + dh)
    check(*dominated(nb, S, H, dh, BF16, (11.2, 12.0), alone, gen), 0.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 400.0])
@pytest.mark.parametrize("nb,S,H,dh", [(1, 64, 2, 64), (1, 150, 2, 128), (24, 150, 24, 64)])
def test_one_visible_key_of_a_large_score(nb, S, H, dh, cap, dtype):
    """Scores of 100 and more: lse, and with it the weight of the only key, is off by more than a unit of 1."""
    gen = torch.Generator().manual_seed(dh)
    k, v, do = (torch.randn(nb, S, H, dh, generator=gen).to(dtype) for _ in range(3))
    q = (k.float() * (100.0 + 60.0 * torch.rand(nb, S, H, 1, generator=gen)) / math.sqrt(dh)).to(dtype)
    docs = torch.arange(S, dtype=torch.int32).view(1, S).expand(nb, S).contiguous()
    got = gradients(q, k, v, do, docs, cap)
    assert torch.equal(got["o"], v)
    assert not got["dq"].any() and not got["dk"].any()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 900.0])
@pytest.mark.parametrize("nb,S,H,order", [(1, 200, 2, "causal"), (13, 200, 20, "causal"), (1, 64, 2, "causal"), (2, 300, 2, "prefix"), (13, 200, 20, "prefix")])
def test_weights_that_vanish_beside_one(nb, S, H, order, cap, dtype):
    """Scores hundreds above all others: the other keys are visible, and their weights are 0 in fp32.  (The prefix ends inside a tile of
    keys, so that a block of keys is whole for queries whose tiles are not.)"""
    gen = torch.Generator().manual_seed(S)
    k, v, do = (torch.randn(nb, S, H, 64, generator=gen).to(dtype) for _ in range(3))
    at = (torch.rand(S, generator=gen) * torch.arange(1, S + 1)).long()      # a key that each query sees
    q = (60.0 * k[:, at].float()).to(dtype)
    compare(q.cuda(), k.cuda(), v.cuda(), do.cuda(), order=order, cap=cap, prefix=torch.full((nb,), 40, dtype=torch.int32) if order == "prefix" else None)
