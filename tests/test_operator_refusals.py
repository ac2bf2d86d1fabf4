"""The calls that take no context refuse bad arguments on the host, before anything is enqueued (no GPU is needed to be refused)."""
import ctypes as C

import pytest
import torch

from paper_2102_03161_amd import binding

FAR = 1 << 20       # an aligned address that nothing reads: every call below is refused first


def description(**over):
    d = dict(dtype=binding.PT_BF16, nb=2, Sq=10, Sk=10, H=4, Hkv=2, dh=64, order=0, q0=0, scale=0.125, cap=0.0)
    d.update(over)
    return binding.PtAttention(**d)


def view(data=FAR, sample=640 * 4, row=64 * 4, head=64):
    return binding.PtHeads(data, sample, row, head)


def forward(a, q=None, k=None, v=None, o=None):
    lib = binding.load_library()
    views = [x if x is not None else view() for x in (q, k, v, o)]
    return lib.pt_attention_fwd(a, *views, None, None), lib.pt_last_error(None).decode()


@pytest.mark.parametrize("over", [dict(dtype=7), dict(nb=-1), dict(Sq=-1), dict(Sk=-2), dict(H=0), dict(Hkv=0), dict(H=3), dict(dh=0), dict(dh=60),
                                  dict(dh=136), dict(Sk=(1 << 18) + 1), dict(Sq=(1 << 18) + 1), dict(q0=-1), dict(q0=1 << 24), dict(order=3),
                                  dict(order=2), dict(k_documents=FAR), dict(q_documents=FAR), dict(scale=0.0), dict(scale=float("nan")),
                                  dict(scale=float("inf")), dict(scale=-1.0), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-40),
                                  dict(nb=1 << 20, Sq=100)],
                         ids=lambda o: "-".join(f"{k}={v}" for k, v in o.items()))
def test_descriptions(over):
    status, message = forward(description(**over))
    assert status == binding.PT_EINVAL and message
    need = C.c_size_t()
    assert binding.load_library().pt_attention_workspace(description(**over), need) == binding.PT_EINVAL


def test_views():
    for name, bad in (("null", view(data=None)), ("aligned", view(data=FAR + 8)), ("sample", view(sample=644)), ("row", view(row=12)), ("head", view(head=4))):
        for at in range(4):
            views = [None] * 4
            views[at] = bad
            status, message = forward(description(), *views)
            assert status == binding.PT_EINVAL and message.startswith("qkvo"[at]), (name, at, message)
    assert forward(description(), o=view(row=0))[0] == binding.PT_EINVAL        # written rows on top of each other
    assert forward(None)[0] == binding.PT_EINVAL
    lib = binding.load_library()
    assert lib.pt_attention_fwd(description(), None, view(), view(), view(), None, None) == binding.PT_EINVAL
    # fp32 rows move in pieces of 4 elements
    assert forward(description(dtype=binding.PT_F32), q=view(row=66))[0] == binding.PT_EINVAL


def test_backward_needs_its_statistics_and_workspace():
    lib, a = binding.load_library(), description()
    need = C.c_size_t()
    assert lib.pt_attention_workspace(a, need) == binding.PT_OK and need.value == 2 * 4 * 10 * 4
    assert lib.pt_attention_workspace(a, None) == binding.PT_EINVAL
    call = lambda lse, ws, n, dk=None: lib.pt_attention_bwd(a, view(), view(), view(), view(), lse, view(), view(), dk or view(), view(), ws, n, None)   # noqa: E731
    assert call(None, FAR, need.value) == binding.PT_EINVAL
    assert call(FAR, None, need.value) == binding.PT_ENOMEM
    assert call(FAR, FAR, need.value - 1) == binding.PT_ENOMEM
    assert call(FAR, FAR + 4, need.value) == binding.PT_EINVAL
    assert call(FAR, FAR, need.value, dk=view(head=0)) == binding.PT_EINVAL


def test_backward_needs_its_statistics_in_fp32_too():
    """fp32 takes no workspace, but reads lse all the same."""
    lib, a = binding.load_library(), description(dtype=binding.PT_F32)
    args = [view()] * 4 + [None] + [view()] * 4
    assert lib.pt_attention_bwd(a, *args, None, 0, None) == binding.PT_EINVAL and b"lse" in lib.pt_last_error(None)


@pytest.mark.parametrize("over", [dict(nb=1 << 30, H=1 << 30, Hkv=1 << 30, Sq=1 << 18), dict(nb=1 << 16, H=1 << 16, Hkv=1, Sq=0), dict(nb=1 << 24, H=1, Hkv=1, Sq=0, Sk=0)],
                         ids=["product past 64 bits", "no queries", "nothing but samples"])
def test_counts_of_heads_that_pass_32_bits(over):
    assert forward(description(**over))[0] == binding.PT_EINVAL


def test_a_cap_that_float_rounds_to_none():
    for cap in (1e-50, -1.0, float("nan")):
        with pytest.raises(binding.PtError):
            binding.AttentionRule(cap=cap)
    with pytest.raises(binding.PtError, match="lse"):
        q = torch.zeros(2, 10, 4, 64, dtype=torch.bfloat16)
        binding.attention_backward(q, q, q, q, None, q)


def test_gelu8():
    lib = binding.load_library()
    f = lambda dtype=1, h=FAR, g=FAR, codes=FAR, exps=FAR, rows=4, F=64: lib.pt_gelu8_fwd(dtype, h, g, codes, exps, rows, F, None)   # noqa: E731
    b = lambda dtype=1, codes=FAR, exps=FAR, dg=FAR, dh=FAR, g=FAR, rows=4, F=64: lib.pt_gelu8_bwd(dtype, codes, exps, dg, dh, g, rows, F, None)   # noqa: E731
    for call in (f, b):
        for bad in (dict(dtype=2), dict(rows=-1), dict(F=0), dict(F=6), dict(F=-4), dict(codes=None), dict(codes=FAR + 4), dict(exps=None), dict(g=FAR + 8),
                    dict(rows=1 << 40)):
            assert call(**bad) == binding.PT_EINVAL, bad
        assert call(rows=0, g=None) == binding.PT_OK        # nothing to do
    assert f(h=None) == f(g=None) == f(h=FAR + 2) == binding.PT_EINVAL
    assert b(dg=None) == b(dh=None) == b(dg=FAR + 2) == b(dh=FAR + 2) == binding.PT_EINVAL


def test_the_binding_refuses_tensors_that_do_not_fit():
    q = torch.zeros(2, 10, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 10, 2, 64, dtype=torch.bfloat16)
    refused = [
        lambda: binding.attention_forward(q, k, k),                                      # not on a GPU
        lambda: binding.attention_forward(q[0], k, k),
        lambda: binding.attention_forward(q, k.float(), k),
        lambda: binding.attention_forward(q, k, k[:, :9]),
        lambda: binding.attention_forward(q.half(), k.half(), k.half()),
        lambda: binding.attention_forward(q.transpose(2, 3), k, k),
        lambda: binding.AttentionRule(order="sideways"),
        lambda: binding.AttentionRule(documents=torch.zeros(2, 10)).describe(q, k),
        lambda: binding.AttentionRule(documents=torch.zeros(10, 2, dtype=torch.int32).T).describe(q, k),
        lambda: binding.AttentionRule(documents=torch.zeros(2, 9, dtype=torch.int32)).describe(q, k),
        lambda: binding.AttentionRule(q_documents=torch.zeros(2, 10, dtype=torch.int32)).describe(q, k),
        lambda: binding.AttentionRule(order="prefix").describe(q, k),
        lambda: binding.AttentionRule(slopes=torch.zeros(3)).describe(q, k),
        lambda: binding.attention_backward(q, k, k, q, torch.zeros(2, 4, 9), q),
        lambda: binding.gelu8_forward(torch.zeros(4, 64)),
        lambda: binding.gelu8_forward(torch.zeros(64)),
        lambda: binding.gelu8_backward(torch.zeros(4, 64), torch.zeros(4, 2), torch.zeros(4, 64)),
    ]
    for at, call in enumerate(refused):
        with pytest.raises(binding.PtError) as e:
            call()
        assert e.value.status == binding.PT_EINVAL, at


def test_checkpoints_shrink_the_work_arena():
    """act8: per token and block the activation and its derivative (2 F elements) become F codes and one exponent for 32 of them,
    and one buffer of F elements serves all blocks."""
    from paper_2102_03161_amd import synth
    for name in ("vit_b16", "bert_base_qa"):
        w = synth.workload(name)
        plain, small = (binding.query_arena_bytes(binding.make_config(w, act8=a)) for a in (False, True))
        T, F, L = w["B"] * w["S"], w["F"], w["L"]
        assert plain[:2] == small[:2] and plain[3] == small[3]
        saved = (L + 1) * 2 * 2 * T * F - (L * T * (F + F // 32) + 2 * T * F)    # the frozen prefix's slot had both as well
        assert abs((plain[2] - small[2]) - saved) <= 4 * 256 * (L + 1)           # rounded up to 256 bytes
    cfg = binding.make_config(w)
    cfg.act8 = 2
    with pytest.raises(binding.PtError):
        binding.query_arena_bytes(cfg)
