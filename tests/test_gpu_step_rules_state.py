"""The training step under a rule: what a change of the rule means to the batch in flight, to cached rows, and across streams."""
import numpy as np
import pytest

from paper_2102_03161_amd import binding, synth
from tests import gpu_harness as H

pytestmark = pytest.mark.gpu


def context(w, seed, **over):
    ctx = binding.Context(binding.make_config(w, **over))
    H.load_params(ctx, H.init_values(w, ctx, seed))
    return ctx


def test_a_rule_set_behind_a_pass_waits_for_the_next_batch():
    import torch
    w = dict(synth.workload("bert_tiny"))
    ctx = context(w, 1)
    x, y = H.batch_for(w, 1, w["B"])
    dx, dy = H.to_dev(torch, x), H.to_dev(torch, y)
    docs = torch.zeros(w["B"], w["S"], dtype=torch.int32, device="cuda")
    docs[:, w["S"] // 2:] = -1
    hk = ctx.frozen_forward(dx)
    plain = ctx.active_fwd_bwd(hk, dy)
    assert ctx.active_fwd_bwd(hk, dy) == plain                       # the same batch again
    for rule in (binding.AttentionRule(documents=docs[:1].contiguous()), binding.AttentionRule(order="causal"), None):
        ctx.set_attention(rule)
        with pytest.raises(binding.PtError) as e:                    # its forward pass was another rule's
            ctx.active_fwd_bwd(hk, dy)
        assert e.value.status == binding.PT_ESTATE
        assert ctx.last_loss() == plain
    norms = ctx.layer_grad_norms()                                   # the pass that is done is still good for an update
    assert np.isfinite(norms).all()
    ctx.set_attention(binding.AttentionRule(documents=docs))
    ctx.optimizer_step(lr=1e-3)
    ruled = ctx.active_fwd_bwd(ctx.frozen_forward(dx), dy)
    assert np.isfinite(ruled) and ruled != plain
    ctx.close()
