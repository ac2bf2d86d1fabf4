"""Attention under a rule at the edges of what its description allows."""
import pytest
import torch

from paper_2102_03161_amd import binding
from tests.rule_reference import check, reference
from tests.test_gpu_attention_rules import BF16, F32, both, compare, inputs

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


@TYPES
def test_padding_against_padding_costs_nothing(dtype):
    """Rows that are nearly all padding take a fraction of the time of full ones (a 64th of the pairs squared, and the list)."""
    nb, S, H = 4, 4096, 8
    gen = torch.Generator().manual_seed(5)
    q, k, v, do = inputs(nb, S, S, H, H, 64, dtype, gen)
    docs = torch.zeros(nb, S, dtype=torch.int32, device="cuda")
    few = docs.clone()
    few[:, 64:] = -1

    def least(rule):
        times = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            o, lse = binding.attention_forward(q, k, v, rule)
            binding.attention_backward(q, k, v, o, lse, do, rule)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    full, padded = least(binding.AttentionRule(documents=docs)), least(binding.AttentionRule(documents=few))
    print(f"full rows {full * 1e3:.0f} us, one tile of each {padded * 1e3:.0f} us", flush=True)
    assert padded < full / 3


def test_documents_of_the_largest_id():
    gen = torch.Generator().manual_seed(6)
    q, k, v, do = inputs(2, 200, 200, 2, 2, 64, BF16, gen)
    docs = torch.full((2, 200), (1 << 31) - 1, dtype=torch.int32)
    docs[0, 60:] = -1
    docs[1, 100:] = 0
    docs[1, 130:] = -(1 << 31)
    compare(q, k, v, do, docs)


@TYPES
@pytest.mark.parametrize("S", [5, 200])
def test_scores_far_below_zero(dtype, S):
    """Every score about -1e31: the only key that a query sees still has all of its weight."""
    gen = torch.Generator().manual_seed(3)
    q, k, v, do = inputs(1, S, S, 2, 2, 64, dtype, gen)
    q, k = torch.full_like(q, 2.0 ** 50), torch.full_like(k, -(2.0 ** 50))
    docs = torch.arange(S, dtype=torch.int32).view(1, S)
    rule = binding.AttentionRule(documents=docs.cuda())
    o, lse = binding.attention_forward(q, k, v, rule)
    assert torch.equal(o, v)
    assert ((lse.double() + 8 * 2.0 ** 100).abs() <= 2.0 ** -21 * 8 * 2.0 ** 100).all()    # -64 2^100 / sqrt(64)


@TYPES
@pytest.mark.parametrize("S", [5, 200])
def test_a_nan_stays_visible(dtype, S):
    """A row of NaN is no row that sees nothing: its statistic and its gradient say so, the other rows have theirs."""
    gen = torch.Generator().manual_seed(4)
    q, k, v, do = (x.clone() for x in inputs(1, S, S, 2, 2, 64, dtype, gen))
    clean = both(q, k, v, do)
    q[:, 3] = float("nan")
    got = both(q, k, v, do)
    rest = torch.arange(S) != 3
    for name in ("o", "dq"):
        assert torch.isnan(got[name][:, 3]).all(), name
        assert torch.equal(got[name][:, rest], clean[name][:, rest]), name
    assert torch.isnan(got["lse"][:, :, 3]).all()
    assert torch.equal(got["lse"][:, :, rest], clean["lse"][:, :, rest])
    assert torch.isnan(got["dk"]).all() and torch.isnan(got["dv"]).all()


@TYPES
def test_prefix_lengths_of_any_value(dtype):
    """A prefix of no or negative length shows nothing more, one behind the end everything."""
    gen = torch.Generator().manual_seed(1)
    lengths = torch.tensor([-(1 << 31), -(1 << 31) + 1, -1, 0, 1, 70, 90, (1 << 31) - 1], dtype=torch.int32)
    q, k, v, do = inputs(len(lengths), 90, 90, 2, 1, 64, dtype, gen)
    compare(q, k, v, do, order="prefix", prefix=lengths)
