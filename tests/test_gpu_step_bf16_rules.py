"""bf16 training steps under a rule and with 8-bit GELU checkpoints, against the oracle with the same attention and the same rounding of
the GELU's input put in.

8e-2 of a tensor's peak (or of the root-sum-square of its summands, where that is larger): how far the rounding of what is stored in bf16
moves gradients at these widths by itself.  A block whose weight gradients read another block's activations, or a mask of another
sample, is off by the size of the gradient."""
import numpy as np
import pytest

from paper_2102_03161_amd import binding, synth
from tests import gpu_harness as H
from tests.test_gpu_parity import MID_BERT, MID_VIT
from tests.test_gpu_step_rules import Rule, labels_on_tokens, patch_checkpoints

pytestmark = pytest.mark.gpu
TOL = 8e-2

CLS = dict(MID_BERT, n_out=5, head="cls")
CASES = {
    "vit act8": (MID_VIT, None, 0, True),
    "bert act8": (MID_BERT, None, 0, True),
    "bert classes act8, frozen": (CLS, None, 1, True),
    "vit cap and slopes": (MID_VIT, dict(cap=4.0, slopes=True), 0, False),
    "vit prefix act8": (MID_VIT, dict(order="prefix"), 1, True),
    "bert padded classes": (CLS, dict(docs="padded"), 0, False),
    "bert packed span, causal, act8": (MID_BERT, dict(docs="packed", order="causal"), 0, True),
    "bert packed classes, prefix, cap": (CLS, dict(docs="packed", order="prefix", cap=6.0), 2, False),
}


@pytest.mark.parametrize("name", list(CASES))
def test_step(monkeypatch, name):
    import torch
    w, over, k, act8 = CASES[name]
    print(f"bf16 step: {name}", flush=True)
    ctx = binding.Context(binding.make_config(w, act8=act8))
    vals = H.init_values(w, ctx, 31)
    if act8:    # first MLP biases of a real model's size, so that blocks hold values of both signs and some spread
        for n in vals:
            if n.endswith(".b1"):
                vals[n] = synth.round_bf16(np.random.default_rng(3).standard_normal(vals[n].shape).astype(np.float32))
    H.load_params(ctx, vals)
    x, y = H.batch_for(w, 31, w["B"])
    if over:
        rule = Rule(w, w["B"], 31, **over)
        y = labels_on_tokens(w, rule, y)
        ctx.set_attention(rule.binding(torch))
    g = H.gpu_step(torch, ctx, w, x, y, k)
    rss = H.summand_rss(w, vals, x, y, k)     # of the step without a rule: sizes
    if over:
        rule.patch(monkeypatch)
    if act8:
        patch_checkpoints(monkeypatch, w, k)
    o = H.oracle_step(w, vals, x, y, k)
    H.oracle_update(w, o, vals, g["grads"], k)
    errs = H.compare_step(w, g, o, k, TOL, rss=rss)
    worst = max(errs.items(), key=lambda kv: kv[1])
    print(f"  worst {worst[0]} = {worst[1]:.3e}", flush=True)
    ctx.close()


@pytest.mark.parametrize("w", [MID_VIT, MID_BERT], ids=["vit", "bert"])
def test_a_checkpointed_step_repeats_and_follows_an_uncheckpointed_one(w):
    """The same step twice gives the same bits; and every gradient of every block points where the step that keeps everything
    points (a cosine of 0.9: rounding may make up four tenths of its norm)."""
    import torch
    grads = []
    for act8 in (True, True, False):
        ctx = binding.Context(binding.make_config(w, act8=act8))
        H.load_params(ctx, H.init_values(w, ctx, 32))
        x, y = H.batch_for(w, 32, w["B"])
        grads.append(H.gpu_step(torch, ctx, w, x, y, 0)["grads"])
        ctx.close()
    first, again, kept = grads
    zero = H.exactly_cancelling(w, 0)
    for name, a in first.items():
        assert np.array_equal(a, again[name]), name
        if name not in zero:
            b = kept[name]
            assert float((a * b).sum()) >= 0.9 * np.linalg.norm(a) * np.linalg.norm(b), name
