"""Attention under a rule on grids that fill the card, where a wave owns its rows alone: every kernel of that kind, against the definition
in 64 bits (tests/rule_reference.py has the bounds)."""
import pytest
import torch

from tests.attention_choice import shares
from tests.test_gpu_attention_rules import BF16, F32, compare, documents, inputs

pytestmark = pytest.mark.gpu

# samples, rows, heads, key heads, head size, order, documents, cap, slopes
BF16_CASES = [
    (13, 200, 20, 20, 64, "full", None, 0.0, False),
    (13, 200, 20, 20, 64, "full", "packed", 8.0, False),
    (13, 200, 20, 20, 64, "causal", "mixed", 0.0, True),
    (13, 200, 20, 20, 40, "prefix", None, 12.0, True),
    (9, 333, 20, 20, 64, "causal", None, 0.0, False),
    (13, 200, 40, 20, 64, "full", "padded", 0.0, False),
    (13, 200, 20, 20, 128, "causal", None, 15.0, False),
    (13, 200, 20, 20, 128, "prefix", "packed", 0.0, False),
    (13, 200, 20, 20, 72, "full", "padded", 9.0, True),
    (13, 200, 20, 10, 128, "full", "packed", 0.0, True),
    (9, 333, 20, 20, 96, "full", None, 0.0, False),
]
F32_CASES = [
    (8, 200, 17, 17, 16, "causal", None, 0.0, True),
    (8, 200, 17, 17, 64, "full", "packed", 7.0, False),
    (6, 333, 16, 16, 128, "prefix", "mixed", 0.0, False),
    (8, 200, 34, 17, 64, "full", "padded", 0.0, True),
    (8, 200, 17, 17, 104, "causal", "packed", 11.0, True),
]


def run(dtype, nb, S, H, Hkv, dh, order, docs, cap, slopes):
    print(f"full grid: {dtype} {nb} {S} {H} {Hkv} {dh} {order} {docs} {cap} {slopes}", flush=True)
    assert set(shares(nb, S, S, H, Hkv, dh, order != "full", docs is not None, bf16=dtype == BF16)) == {1}
    gen = torch.Generator().manual_seed(S * 17 + dh + H)
    q, k, v, do = inputs(nb, S, S, H, Hkv, dh, dtype, gen, "packed" if S % 2 else "heads")
    compare(q, k, v, do, documents(docs, nb, S, gen), order=order, cap=cap, slopes=torch.rand(H, generator=gen) * 0.3 if slopes else None,
            prefix=torch.randint(0, S + 1, (nb,), generator=gen).int() if order == "prefix" else None)


@pytest.mark.parametrize("case", BF16_CASES, ids=lambda c: "-".join(map(str, c)))
def test_bf16(case):
    run(BF16, *case)


@pytest.mark.parametrize("case", F32_CASES, ids=lambda c: "-".join(map(str, c)))
def test_f32(case):
    run(F32, *case)


def test_one_query_of_many_heads():
    """One query a head over long rows of keys, forward and back."""
    gen = torch.Generator().manual_seed(3)
    assert shares(27, 1, 4100, 19, 19, 8, False, True) == (1, 1, 1)
    q, k, v, do = inputs(27, 1, 4100, 19, 19, 8, BF16, gen)
    docs = documents("packed", 27, 4100, gen)
    compare(q, k, v, do, docs, docs[:, :1].contiguous())
