"""Attention under a rule at the edges of what its description allows."""
import pytest
import torch

from paper_2102_03161_amd import binding
from tests.rule_reference import check, reference
from tests.test_gpu_attention_rules import BF16, F32, both, inputs

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@TYPES
@pytest.mark.parametrize("order,S", [("full", 64), ("causal", 64), ("full", 50), ("full", 7)])
def test_a_sample_alone_and_among_others(dtype, order, S):
    """Few pairs a sample: the same bits whatever the batch, on a grid below the number of CUs and on one far above."""
    gen = torch.Generator().manual_seed(2)
    nb, H = 45, 16
    q, k, v, do = inputs(nb, S, S, H, H, 64, dtype, gen)
    rule = dict(order=order, cap=20.0 if S == 50 else 0.0)
    whole = both(q, k, v, do, **rule)
    one = slice(7, 8)
    alone = both(q[one], k[one], v[one], do[one], **rule)
    for name in whole:
        if dtype == BF16:
            assert torch.equal(whole[name][one], alone[name]), name
    want = reference(q[one], k[one], v[one], do[one], few=dtype == BF16, **rule)
    for name in want:
        check(name, whole[name][one], want[name])
