"""The training step with attention under a rule and with 8-bit GELU checkpoints, against the oracle with the same attention, the
same padding in its span loss, or the same rounding of the GELU's input put in."""
import numpy as np
import pytest
from scipy.special import erf

from oracle import encoder as orc
from paper_2102_03161_amd import binding, synth
from tests import gpu_harness as H
from tests.test_gpu_gelu8 import pack, unpack
from tests.test_gpu_parity import MID_BERT, MID_VIT

pytestmark = pytest.mark.gpu
TOL = 1e-4      # the fp32 bar of the parity tests


class Rule:
    """A rule in numpy, and as the binding takes it; `rows`: which samples of the arrays a batch holds."""

    def __init__(self, w, n, seed, order="full", cap=0.0, slopes=False, docs=None):
        rng = np.random.default_rng(seed)
        S = w["S"]
        self.order, self.cap = order, cap
        self.slopes = rng.uniform(0.0, 0.3, w["H"]).astype(np.float32) if slopes else None
        self.prefix = rng.integers(0, S, n).astype(np.int32) if order == "prefix" else None
        self.docs = None
        if docs:
            used = rng.integers(S // 2, S + 1, n)
            self.docs = np.zeros((n, S), np.int32)
            if docs == "packed":
                cut = rng.integers(1, S // 2, n)
                self.docs[np.arange(S)[None] >= cut[:, None]] = 1
            self.docs[np.arange(S)[None] >= used[:, None]] = -1

    def binding(self, torch, rows=slice(None)):
        dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a[rows] if a.ndim > 1 or a is self.prefix else a)).cuda()   # noqa: E731
        return binding.AttentionRule(order=self.order, cap=self.cap, slopes=dev(self.slopes), documents=dev(self.docs), prefix=dev(self.prefix))

    def patch(self, monkeypatch):
        """The oracle's attention and span loss under this rule (for batches of all n samples)."""
        def probabilities(cfg, q, k):
            B, _, S, dh = q.shape
            t = (q @ k.transpose(0, 1, 3, 2)) / np.sqrt(dh)
            bent = np.tanh(t / self.cap) if self.cap else np.zeros_like(t)
            s = self.cap * bent if self.cap else t
            i, j = np.arange(S)[:, None], np.arange(S)[None, :]
            if self.slopes is not None:
                s = s - self.slopes.astype(np.float64)[None, :, None, None] * np.abs(i - j)
            see = np.ones((B, 1, S, S), bool)
            if self.order != "full":
                see &= (j <= i)[None, None]
            if self.order == "prefix":
                see |= (j[None] < self.prefix[:B, None, None])[:, None]
            if self.docs is not None:
                d = self.docs[:B]
                see &= ((d[:, :, None] == d[:, None, :]) & (d[:, :, None] >= 0))[:, None]
            s = np.where(see, s, -np.inf)
            top = s.max(-1, keepdims=True)
            e = np.exp(s - np.where(np.isinf(top), 0.0, top))
            total = e.sum(-1, keepdims=True)
            return e / np.where(total == 0, 1.0, total), 1.0 - bent * bent

        def forward(cfg, p, pre, xin):
            D = cfg.D
            qkv = xin @ p[pre + "Wqkv"] + p[pre + "bqkv"]
            q, k, v = (orc._split_heads(qkv[..., n * D:(n + 1) * D], cfg.H) for n in range(3))
            P, slope = probabilities(cfg, q, k)
            c = orc._merge_heads(P @ v)
            return c @ p[pre + "Wo"] + p[pre + "bo"], (xin, q, k, v, P, slope, c)

        def backward(cfg, p, pre, da, saved, grads):
            xin, q, k, v, P, slope, c = saved
            D, dh = cfg.D, cfg.D // cfg.H
            grads[pre + "Wo"] = c.reshape(-1, D).T @ da.reshape(-1, D)
            grads[pre + "bo"] = da.sum(axis=(0, 1))
            dc = orc._split_heads(da @ p[pre + "Wo"].T, cfg.H)
            dv = P.transpose(0, 1, 3, 2) @ dc
            dP = dc @ v.transpose(0, 1, 3, 2)
            dS = P * (dP - (dP * P).sum(axis=-1, keepdims=True)) * slope / np.sqrt(dh)
            dqkv = np.concatenate([orc._merge_heads(x) for x in (dS @ k, dS.transpose(0, 1, 3, 2) @ q, dv)], axis=-1)
            grads[pre + "Wqkv"] = xin.reshape(-1, D).T @ dqkv.reshape(-1, 3 * D)
            grads[pre + "bqkv"] = dqkv.sum(axis=(0, 1))
            return dqkv @ p[pre + "Wqkv"].T

        monkeypatch.setattr(orc, "mhsa_forward", forward)
        monkeypatch.setattr(orc, "mhsa_backward", backward)
        if self.docs is not None:
            real = orc.head_loss_forward

            def loss(cfg, p, xL, labels):
                if cfg.arch == "vit" or cfg.head == "cls":
                    return real(cfg, p, xL, labels)
                z = xL @ p["head.W"] + p["head.b"]
                zt = np.where(self.docs[:, None, :] >= 0, z.transpose(0, 2, 1), -np.inf)
                prob = orc.softmax_lastaxis(zt)
                B = len(labels)
                picked = np.stack([prob[np.arange(B), c, labels[:, c]] for c in range(2)], axis=1)
                return (-0.5 * np.log(picked).sum(axis=1)).mean(), z, (xL, prob, np.asarray(labels))

            monkeypatch.setattr(orc, "head_loss_forward", loss)


def labels_on_tokens(w, rule, y):
    """Span labels moved onto tokens that are no padding."""
    if rule.docs is None or w["arch"] == "vit" or w.get("head") == "cls":
        return y
    used = (rule.docs >= 0).sum(1)
    return (y % used[:, None]).astype(y.dtype)


CASES = {
    "vit cap and slopes": (dict(synth.workload("vit_tiny")), dict(cap=4.0, slopes=True), 0),
    "vit prefix, frozen": (dict(MID_VIT, dtype="f32"), dict(order="prefix", cap=20.0), 1),
    "bert padded span": (dict(synth.workload("bert_tiny")), dict(docs="padded"), 0),
    "bert packed span, causal": (dict(MID_BERT, dtype="f32"), dict(docs="packed", order="causal"), 0),
    "bert padded classes": (dict(synth.workload("bert_tiny_cls")), dict(docs="padded", slopes=True), 1),
    "bert padded classes, all frozen": (dict(synth.workload("bert_tiny_cls")), dict(docs="padded"), 2),
}


@pytest.mark.parametrize("act8", [False, True], ids=["kept", "act8"])
@pytest.mark.parametrize("name", list(CASES))
def test_step_under_a_rule(monkeypatch, name, act8):
    import torch
    w, over, k = CASES[name]
    print(f"step under a rule: {name} act8={act8}", flush=True)
    rule = Rule(w, w["B"], 21, **over)
    ctx = binding.Context(binding.make_config(w, act8=act8))
    vals = H.init_values(w, ctx, 21)
    if act8:    # first MLP biases of a real model's size, so that blocks hold values of both signs and some spread
        for n in vals:
            if n.endswith(".b1"):
                vals[n] = np.random.default_rng(3).standard_normal(vals[n].shape).astype(np.float32)
    H.load_params(ctx, vals)
    x, y = H.batch_for(w, 21, w["B"])
    y = labels_on_tokens(w, rule, y)
    ctx.set_attention(rule.binding(torch))
    g = H.gpu_step(torch, ctx, w, x, y, k)
    rule.patch(monkeypatch)
    if act8:
        patch_checkpoints(monkeypatch, w, k)
    o = H.oracle_step(w, vals, x, y, k)
    H.oracle_update(w, o, vals, g["grads"], k)
    # act8: a code may fall on the other side of a tie between the oracle's input and the kernels', which differs by 1e-6 or so.
    # Per value the chance is 1e-6 over a step (about 2e-2): a few values of a block, each off by one step: 1/100 of the largest
    # value of its row of 32, in a sum over a hundred tokens or more
    H.compare_step(w, g, o, k, 5e-3 if act8 else TOL)
    ctx.set_attention(None)
    plain = H.gpu_step(torch, ctx, w, x, y, k)
    assert abs(plain["loss"] - g["loss"]) > 1e-7 * abs(g["loss"])       # the rule made a difference
    ctx.close()


def patch_checkpoints(monkeypatch, w, k):
    """The oracle's MLP backward pass from the rounded pre-activation; the top block under a first-token head keeps its own."""
    top = w["L"] - 1 if H.first_token_rows_only(w, k) else None
    back = orc.mlp_backward

    def backward(cfg, p, pre, dout, saved, grads):
        xin, h, g = saved
        if pre != f"blk{top}.":
            flat = h.reshape(-1, h.shape[-1])
            h = unpack(*pack(flat)).reshape(h.shape)
            g = 0.5 * h * (1.0 + erf(h / np.sqrt(2.0)))
        return back(cfg, p, pre, dout, (xin, h, g), grads)

    monkeypatch.setattr(orc, "mlp_backward", backward)


@pytest.mark.parametrize("dtype,tol", [("f32", TOL), ("bf16", 8e-2)])
def test_a_padded_batch_trains_like_the_sequences_without_padding(dtype, tol):
    """A row of 40 tokens and 32 of padding against a row of 40: the loss and every gradient.  (bf16: 8e-2 is how far the rounding
    of what is stored moves gradients at such widths by itself.)"""
    import torch
    long = dict(MID_BERT, dtype=dtype, S=72)
    short = dict(long, S=40)
    a, b = binding.Context(binding.make_config(long)), binding.Context(binding.make_config(short))
    vals = H.init_values(long, a, 5)
    H.load_params(a, vals)
    H.load_params(b, vals)
    x, y = H.batch_for(short, 5, short["B"])
    wide = np.full((long["B"], 72), 7, np.int32)
    wide[:, :40] = x
    docs = np.full((long["B"], 72), -1, np.int32)
    docs[:, :40] = 0
    a.set_attention(binding.AttentionRule(documents=torch.from_numpy(docs).cuda()))
    ga = H.gpu_step(torch, a, long, wide, y, 0)
    gb = H.gpu_step(torch, b, short, x, y, 0)
    assert abs(ga["loss"] - gb["loss"]) <= tol * abs(gb["loss"])
    for name in ga["grads"]:
        peak = np.abs(gb["grads"][name]).max()
        if name not in H.exactly_cancelling(long, 0):
            assert np.abs(ga["grads"][name] - gb["grads"][name]).max() <= tol * peak, name
    a.close()
    b.close()


def test_cached_rows_in_any_order_follow_their_documents():
    """A batch whose samples are cached at different boundaries is computed in another order than it was given in: every sample
    keeps its own documents."""
    import torch
    w = dict(MID_BERT, dtype="f32")
    rule = Rule(w, w["B"], 8, docs="packed", order="prefix")
    x, y = H.batch_for(w, 8, w["B"])
    y = labels_on_tokens(w, rule, y)
    ref, ctx = (binding.Context(binding.make_config(w, cache_slots=8)) for _ in range(2))
    vals = H.init_values(w, ctx, 8)
    for c in (ref, ctx):
        H.load_params(c, vals)
        c.set_attention(rule.binding(torch))
    ids = np.arange(w["B"])
    ctx.set_freeze_boundary(1)
    late = [3, 0]          # two samples get rows at boundary 1, under their own documents
    ctx.set_attention(rule.binding(torch, late))
    ctx.frozen_forward(H.to_dev(torch, x[late]), ids[late])
    ctx.active_fwd_bwd(ctx.frozen_forward(H.to_dev(torch, x[late]), ids[late]), H.to_dev(torch, y[late]))
    ctx.set_attention(rule.binding(torch))
    for c in (ref, ctx):
        c.set_freeze_boundary(2)
    want = H.gpu_step(torch, ref, w, x, y, 2)
    got = H.gpu_step(torch, ctx, w, x, y, 2, sample_ids=ids)     # two advances, three misses
    assert ctx.cache_stats()["advances"] == 2
    assert np.array_equal(want["hk"], got["hk"])
    assert want["loss"] == got["loss"]
    ref.close()
    ctx.close()


def test_a_label_on_padding_counts_nothing():
    import torch
    w = dict(synth.workload("bert_tiny"))
    docs = np.zeros((w["B"], w["S"]), np.int32)
    docs[:, 10:] = -1
    docs[0] = -1
    x, y = H.batch_for(w, 4, w["B"])
    y = (y % 10).astype(np.int32)
    y[1] = 12                                       # both labels of sample 1 on padding; sample 0 has nothing else
    ctx = binding.Context(binding.make_config(w))
    H.load_params(ctx, H.init_values(w, ctx, 4))
    ctx.set_attention(binding.AttentionRule(documents=torch.from_numpy(docs).cuda()))
    all_four = H.gpu_step(torch, ctx, w, x, y, 0)
    assert np.isfinite(all_four["loss"])
    assert all(np.isfinite(a).all() for a in all_four["grads"].values())
    other = binding.Context(binding.make_config(w))
    H.load_params(other, H.init_values(w, other, 4))
    other.set_attention(binding.AttentionRule(documents=torch.from_numpy(docs[2:]).cuda()))
    two = H.gpu_step(torch, other, w, x[2:], y[2:], 0)
    assert abs(all_four["loss"] * 4 - two["loss"] * 2) <= TOL * two["loss"]      # the mean is over all four
    for name, a in all_four["grads"].items():
        if name not in H.exactly_cancelling(w, 0):
            assert np.abs(2 * a - two["grads"][name]).max() <= TOL * np.abs(two["grads"][name]).max(), name
    ctx.close()
    other.close()


def test_refusals_and_call_order():
    import torch
    w = dict(synth.workload("bert_tiny"))
    ctx = binding.Context(binding.make_config(w))
    H.load_params(ctx, H.init_values(w, ctx, 1))
    x, y = H.batch_for(w, 1, w["B"])
    docs = torch.zeros(w["B"] - 1, w["S"], dtype=torch.int32, device="cuda")
    for bad in (dict(order="prefix"), dict(cap=-1.0), dict(cap=float("nan")), dict(scale=0.5), dict(q0=1),
                dict(documents=docs[:, :-1].contiguous()), dict(documents=docs.cpu()), dict(slopes=torch.zeros(1, device="cuda")),
                dict(documents=torch.zeros(w["B"] + 1, w["S"], dtype=torch.int32, device="cuda"))):
        with pytest.raises(binding.PtError) as e:
            ctx.set_attention(binding.AttentionRule(**bad))
        assert e.value.status == binding.PT_EINVAL, bad
    ctx.set_attention(binding.AttentionRule(documents=docs))
    with pytest.raises(binding.PtError) as e:       # more samples than the rule describes
        ctx.frozen_forward(H.to_dev(torch, x), None)
    assert e.value.status == binding.PT_EINVAL
    hk = ctx.frozen_forward(H.to_dev(torch, x[:3]), None)
    with pytest.raises(binding.PtError) as e:
        ctx.set_attention(None)
    assert e.value.status == binding.PT_ESTATE
    assert np.isfinite(ctx.active_fwd_bwd(hk, H.to_dev(torch, y[:3])))
    ctx.set_attention(None)
    ctx.close()
