"""Contexts with 8-bit GELU checkpoints: more values than their kernels count are refused where the context is planned."""
import pytest

from paper_2102_03161_amd import binding, synth


def test_more_values_than_the_kernels_count():
    w = dict(synth.workload("bert_tiny"), S=512, max_pos=512, F=8192)
    most = (1 << 27) // (8192 // 32) // 512
    for act8 in (False, True):
        binding.query_arena_bytes(binding.make_config(dict(w, B=most), act8=act8))
    binding.query_arena_bytes(binding.make_config(dict(w, B=most + 1)))
    with pytest.raises(binding.PtError) as e:
        binding.query_arena_bytes(binding.make_config(dict(w, B=most + 1), act8=True))
    assert e.value.status == binding.PT_EINVAL
