"""Written views whose rows or heads would lie on top of each other are refused on the host (no GPU is needed to be refused)."""
import ctypes as C

import pytest

from paper_2102_03161_amd import binding
from tests.test_operator_refusals import FAR, description, view

OVERLAPS = [dict(row=0), dict(row=8), dict(row=56), dict(row=-56), dict(head=0), dict(head=32), dict(head=-8), dict(sample=0), dict(sample=16)]


@pytest.mark.parametrize("over", OVERLAPS, ids=lambda o: "-".join(f"{k}={v}" for k, v in o.items()))
def test_outputs_on_top_of_each_other(over):
    lib, a, bad = binding.load_library(), description(), view(**over)
    assert lib.pt_attention_fwd(a, view(), view(), view(), bad, None, None) == binding.PT_EINVAL
    assert lib.pt_last_error(None).startswith(b"o is written")
    need = C.c_size_t()
    assert lib.pt_attention_workspace(a, need) == binding.PT_OK
    for at, name in enumerate(("dq", "dk", "dv")):
        grads = [view(), view(), view()]
        grads[at] = bad
        assert lib.pt_attention_bwd(a, view(), view(), view(), view(), FAR, view(), *grads, FAR, need.value, None) == binding.PT_EINVAL
        assert lib.pt_last_error(None).startswith(name.encode() + b" is written")


def test_the_workspace_of_both_types():
    lib, need = binding.load_library(), C.c_size_t()
    for dtype, values in ((binding.PT_BF16, 1), (binding.PT_F32, 2)):
        assert lib.pt_attention_workspace(description(dtype=dtype), need) == binding.PT_OK and need.value == 2 * 4 * 10 * 4 * values
        args = [view()] * 4 + [FAR] + [view()] * 4
        assert lib.pt_attention_bwd(description(dtype=dtype), *args, FAR, need.value - 1, None) == binding.PT_ENOMEM
