"""Attention under a rule against the definition in 64 bits (tests/rule_reference.py has the bounds)."""
import pytest
import torch

from paper_2102_03161_amd import binding
from tests.rule_reference import check, reference

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def documents(kind, nb, S, gen):
    if kind is None:
        return None
    d = torch.zeros(nb, S, dtype=torch.int32)
    for b in range(nb):
        used = S if kind == "mixed" else int(torch.randint(1, S + 1, (1,), generator=gen))
        if kind == "packed":
            cuts = torch.randint(0, used, (3,), generator=gen)
            d[b] = (torch.arange(S).view(-1, 1) >= cuts.view(1, -1)).sum(1).int()
        if kind == "mixed":      # in no order, padding in between
            d[b] = torch.randint(-1, 4, (S,), generator=gen).int()
        d[b, used:] = -1
    return d


def inputs(nb, Sq, Sk, H, Hkv, dh, dtype, gen, layout="packed"):
    r = lambda *s: torch.randn(*s, generator=gen)   # noqa: E731
    if layout == "packed" and Sq == Sk:
        x = (1.3 * r(nb, Sq, H + 2 * Hkv, dh)).to(dtype).cuda()
        q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    else:
        q = (1.3 * r(nb, H, Sq, dh)).to(dtype).cuda().transpose(1, 2)
        k, v = ((1.3 * r(nb, Hkv, Sk, dh)).to(dtype).cuda().transpose(1, 2) for _ in range(2))
    return q, k, v, r(nb, Sq, H, dh).to(dtype).cuda()


def both(q, k, v, do, docs=None, q_docs=None, **rule):
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    r = binding.AttentionRule(order=rule.get("order", "full"), scale=rule.get("scale"), cap=rule.get("cap", 0.0), slopes=dev(rule.get("slopes")),
                              documents=dev(docs), q_documents=dev(q_docs), prefix=dev(rule.get("prefix")), q0=rule.get("q0", 0))
    o, lse = binding.attention_forward(q, k, v, r)
    dq, dk, dv = binding.attention_backward(q, k, v, o, lse, do, r)
    torch.cuda.synchronize()
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


def compare(q, k, v, do, docs=None, q_docs=None, **rule):
    want = reference(q, k, v, do, q_docs=docs if q_docs is None else q_docs, k_docs=docs, **rule)
    got = both(q, k, v, do, docs, q_docs, **rule)
    for name in want:
        check(name, got[name], want[name])
    return got


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nb,S,H,Hkv,dh,order,docs,cap,slopes", [
    (1, 1, 1, 1, 8, "full", None, 0, False),
    (2, 2, 3, 1, 16, "causal", "packed", 0, True),
    (3, 17, 4, 4, 24, "full", "mixed", 5.0, False),
    (1, 63, 2, 2, 64, "prefix", None, 0, False),
    (2, 64, 2, 1, 64, "full", "padded", 0, False),
    (1, 65, 4, 2, 72, "causal", None, 20.0, True),
    (2, 129, 3, 3, 64, "full", "packed", 0, True),
    (2, 200, 6, 2, 128, "prefix", "packed", 30.0, False),
    (1, 257, 2, 2, 40, "causal", "mixed", 0, False),
    (2, 384, 2, 2, 64, "full", None, 0, False),
    (1, 511, 2, 1, 96, "prefix", "packed", 15.0, True),
    (1, 640, 1, 1, 64, "causal", "packed", 0, False),
])
def test_both_directions_match_the_definition(dtype, nb, S, H, Hkv, dh, order, docs, cap, slopes):
    print(f"attention rule: {dtype} {nb} {S} {H} {Hkv} {dh} {order} {docs} {cap} {slopes}", flush=True)
    gen = torch.Generator().manual_seed(S * 131 + dh)
    q, k, v, do = inputs(nb, S, S, H, Hkv, dh, dtype, gen, "packed" if S % 2 else "heads")
    compare(q, k, v, do, documents(docs, nb, S, gen), order=order, cap=float(cap), slopes=torch.rand(H, generator=gen) * 0.3 if slopes else None,
            prefix=torch.randint(0, S + 1, (nb,), generator=gen).int() if order == "prefix" else None)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Sq,Sk,q0,order", [(1, 300, 0, "full"), (1, 513, 512, "causal"), (5, 131, 126, "causal"), (70, 300, 100, "prefix"), (130, 7, 0, "full"), (3, 40, 90, "causal")])
def test_queries_and_keys_of_different_numbers(dtype, Sq, Sk, q0, order):
    print(f"attention rule: {dtype} {Sq} queries at {q0}, {Sk} keys, {order}", flush=True)
    gen = torch.Generator().manual_seed(Sq + Sk)
    q, k, v, do = inputs(2, Sq, Sk, 4, 2, 64, dtype, gen)
    docs = documents("packed", 2, Sk, gen)
    q_docs = torch.randint(-1, 3, (2, Sq), generator=gen).int()
    compare(q, k, v, do, docs, q_docs, order=order, q0=q0, prefix=torch.tensor([-3, Sk + 9], dtype=torch.int32) if order == "prefix" else None)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_padding_may_hold_anything_and_gets_zeros(dtype):
    gen = torch.Generator().manual_seed(5)
    nb, S, H, dh = 3, 150, 2, 64
    q, k, v, do = (x.clone() for x in inputs(nb, S, S, H, H, dh, dtype, gen))
    docs = documents("packed", nb, S, gen)
    docs[1] = -1                  # a sample of padding alone
    docs[0, 40:44] = -1           # padding in the middle
    pad = (docs < 0).cuda()
    clean = both(q, k, v, do, docs)
    for x, bad in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (do, -float("inf"))):
        x[pad] = bad
    got = compare(q, k, v, do, docs)
    for name in ("o", "dq", "dk", "dv"):
        assert torch.equal(got[name], clean[name]), name
        assert (got[name][pad] == 0).all(), name
    assert torch.isinf(got["lse"].transpose(1, 2)[pad]).all()


@pytest.mark.parametrize("cap,slopes", [(0.0, False), (15.0, False), (50.0, True), (0.0, True)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_a_query_that_sees_one_key_copies_its_value_and_has_no_gradient(dtype, cap, slopes):
    gen = torch.Generator().manual_seed(6)
    rule = dict(cap=cap, slopes=torch.tensor([0.1, 0.4]) if slopes else None)
    for nb, S, docs in ((50, 1, None), (1, 70, torch.arange(70, dtype=torch.int32).view(1, -1))):
        q, k, v, do = inputs(nb, S, S, 2, 2, 64, dtype, gen)
        got = both(q, k, v, do, docs, **rule)
        assert torch.equal(got["o"], v)
        # the probability itself comes from the row's statistic again: e^(s - lse), where s and lse, of size up to cap (or 12 without
        # one), are each a few fp32 roundings (16 of cap + |s| for the capped score, 8 of |lse|); bf16 rounds that away
        off = 0.0 if dtype == BF16 else 2.0 ** -24 * (2 * 16 * 2 * (cap or 12.0) + 8 * (cap or 12.0))
        assert ((got["dv"] - do).abs() <= off * do.abs()).all()
        assert not got["dq"].any() and not got["dk"].any()
    # the last key alone in its document, seen by a tile of queries that see nothing else
    q, k, v, do = inputs(1, 64, 33, 2, 2, 64, dtype, gen)
    docs = torch.zeros(1, 33, dtype=torch.int32)
    docs[0, 32] = 1
    got = both(q, k, v, do, docs, torch.ones(1, 64, dtype=torch.int32), **rule)
    assert torch.equal(got["o"], v[:, 32:].expand(1, 64, 2, 64))
    assert not got["dq"].any() and not got["dk"].any()


def test_views_of_any_strides_and_broadcast_keys():
    gen = torch.Generator().manual_seed(7)
    nb, S, H, dh = 2, 90, 4, 64
    wide = torch.randn(S, nb, 2, H, 3 * dh, generator=gen).to(BF16).cuda()      # rows outermost, heads 3 dh apart
    q = wide[:, :, 0, :, dh:2 * dh].transpose(0, 1)
    k = wide[:, :1, 1, :1, :dh].transpose(0, 1).expand(nb, S, H, dh)            # one key head for every sample and head
    v = wide[:, :, 1, :, 2 * dh:].transpose(0, 1).flip(0)
    do = torch.randn(nb, H, S, dh, generator=gen).to(BF16).cuda().transpose(1, 2)
    want = reference(q, k, v, do, order="causal")
    rule = binding.AttentionRule(order="causal")
    room = torch.full((nb, S, 3, H, dh), 7.0, dtype=BF16, device="cuda")        # outputs side by side in one tensor
    out = torch.full((nb, S + 1, H, dh), 7.0, dtype=BF16, device="cuda")
    o, lse = binding.attention_forward(q, k, v, rule, out=out[:, :S])
    binding.attention_backward(q, k, v, o, lse, do, rule, grads=tuple(room[:, :, x] for x in range(3)))
    for name, got in (("o", o), ("lse", lse), ("dq", room[:, :, 0]), ("dk", room[:, :, 1]), ("dv", room[:, :, 2])):
        check(name, got, want[name])
    assert (out[:, S] == 7).all()        # the row behind the last is left as it was


def test_offsets_beyond_32_bits():
    gen = torch.Generator().manual_seed(8)
    S, far = 600, 1 << 22                # 600 rows 2^22 elements apart: 2.5e9 elements
    room = torch.empty(S * far, dtype=BF16, device="cuda")
    kv = room.view(1, S, far)[:, :, :256].view(1, S, 4, 64)
    kv.copy_(torch.randn(1, S, 4, 64, generator=gen))
    q, do = (torch.randn(1, S, 2, 64, generator=gen).to(BF16).cuda() for _ in range(2))
    compare(q, kv[:, :, :2], kv[:, :, 2:], do, order="causal")


def test_documents_far_apart_in_a_long_row():
    gen = torch.Generator().manual_seed(9)
    S = 5000                              # more tiles than one round of the list holds
    docs = (torch.arange(S) // 700).int().view(1, -1)
    docs[0, 4300:] = 0                    # the first document goes on at the end
    q, k, v, do = inputs(1, S, S, 1, 1, 64, BF16, gen)
    compare(q, k, v, do, docs)


def test_the_longest_row():
    """2^18 keys, 4096 tiles: a few queries at its end, a document that starts where the row does and one that ends there."""
    gen = torch.Generator().manual_seed(12)
    Sk, Sq = 1 << 18, 40
    q, k, v, do = inputs(1, Sq, Sk, 1, 1, 16, BF16, gen)
    docs = torch.zeros(1, Sk, dtype=torch.int32)
    docs[0, 100000:] = 1
    q_docs = torch.ones(1, Sq, dtype=torch.int32)
    q_docs[0, :7] = 0
    compare(q, k, v, do, docs, q_docs, order="causal", q0=Sk - Sq)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_more_workgroups_than_the_gpu_has_cus(dtype):
    gen = torch.Generator().manual_seed(13)
    q, k, v, do = inputs(8, 260, 260, 8, 8, 32, dtype, gen)
    compare(q, k, v, do, documents("packed", 8, 260, gen), order="prefix", prefix=torch.arange(8, dtype=torch.int32) * 30, cap=12.0)


@pytest.mark.parametrize("dtype,dh", [(BF16, 64), (BF16, 128), (F32, 128)], ids=["bf16 64", "bf16 128", "f32 128"])
def test_results_repeat_bit_for_bit_on_any_stream_and_in_a_graph(dtype, dh):
    gen = torch.Generator().manual_seed(10)
    q, k, v, do = inputs(4, 300, 300, 4, 2, dh, dtype, gen)
    docs = documents("packed", 4, 300, gen)
    first = both(q, k, v, do, docs, cap=10.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both(q, k, v, do, docs, cap=10.0)
    for name in first:
        assert torch.equal(first[name], again[name]), name
    rule = binding.AttentionRule(cap=10.0, documents=docs.cuda())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = binding.attention_forward(q, k, v, rule)
        grads = binding.attention_backward(q, k, v, o, lse, do, rule)
    for step in range(3):
        q.copy_((torch.randn(q.shape, generator=gen)).to(dtype))
        graph.replay()
        torch.cuda.synchronize()
        want = both(q, k, v, do, docs, cap=10.0)
        for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
            assert torch.equal(got, want[name]), (step, name)


def test_gradients_agree_with_differences():
    """fp32: the loss sum(o * w) at two points 2 h apart along a random direction; the difference is off by the third order (h^2)
    and by the loss's rounding over h."""
    gen = torch.Generator().manual_seed(11)
    q, k, v, do = inputs(2, 33, 33, 2, 2, 16, F32, gen)
    docs = documents("packed", 2, 33, gen)
    rule = dict(cap=8.0, slopes=torch.tensor([0.1, 0.4]))
    got = both(q, k, v, do, docs, **rule)
    loss = lambda a, b, c: float((both(a, b, c, do, docs, **rule)["o"].double() * do.double()).sum())   # noqa: E731
    h = 2.0 ** -7
    for at, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(q.shape, generator=gen).cuda()
        x = [q, k, v]
        up, down = list(x), list(x)
        up[at], down[at] = x[at] + h * way, x[at] - h * way
        slope = (loss(*up) - loss(*down)) / (2 * h)
        exact = float((got[name].double() * way.double()).sum())
        size = float((got[name].double().abs() * way.double().abs()).sum())
        # rounding: 2^-22 of the loss's terms (about |o||do| of 2112 values) over 2 h; third order: h^2 of the gradient's size
        assert abs(slope - exact) <= 3 * h * h * size + 2112 * 2.0 ** -22 / (2 * h), name


def test_lengths_of_zero():
    for nb, Sq, Sk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        q = torch.randn(nb, Sq, 2, 64, device="cuda").to(BF16)
        k, v = (torch.randn(nb, Sk, 2, 64, device="cuda").to(BF16) for _ in range(2))
        got = both(q, k, v, torch.ones_like(q))
        for name in ("o", "dq", "dk", "dv"):
            assert not got[name].any(), (name, nb, Sq, Sk)
        assert (got["lse"] == -float("inf")).all()


@pytest.mark.parametrize("cap,order,S", [(0.0, "full", 64), (20.0, "causal", 64), (0.0, "prefix", 33), (0.0, "full", 3)])
def test_few_pairs_keep_what_rounding_their_weights_leaves_out(cap, order, S):
    gen = torch.Generator().manual_seed(77)
    q, k, v, do = inputs(2, S, S, 4, 2, 64, BF16, gen)
    rule = dict(order=order, cap=cap, prefix=torch.tensor([5, 20], dtype=torch.int32) if order == "prefix" else None)
    want, got = reference(q, k, v, do, few=True, **rule), both(q, k, v, do, **rule)
    for name in want:
        check(name, got[name], want[name])
