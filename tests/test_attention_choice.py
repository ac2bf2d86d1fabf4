"""How many waves share the rows that a wave owns alone otherwise, at the borders of the rule."""
from tests.attention_choice import shares


def test_bf16_heads_of_64():
    rows = dict(Sq=200, Sk=200, dh=64)                        # two blocks of 128 rows a head
    assert shares(1, H=127, Hkv=127, **rows) == (2, 2, 2)
    assert shares(1, H=128, Hkv=128, **rows) == (2, 1, 1)     # 256 blocks, one for each CU
    assert shares(1, H=256, Hkv=256, **rows) == (2, 1, 1)
    assert shares(1, H=257, Hkv=257, **rows) == (1, 1, 1)
    assert shares(1, H=256, Hkv=256, ordered=True, **rows) == (2, 2, 2)
    assert shares(1, H=257, Hkv=257, ordered=True, **rows) == (1, 1, 1)
    assert shares(1, H=256, Hkv=256, ordered=True, documents=True, **rows) == (2, 1, 1)
    assert shares(8, H=40, Hkv=8, **rows) == (1, 1, 2)        # key heads are fewer


def test_bf16_wider_heads():
    rows = dict(Sq=200, Sk=200, dh=72)
    assert shares(1, H=127, Hkv=127, **rows) == (2, 2, 2)
    assert shares(1, H=128, Hkv=128, **rows) == (1, 1, 1)
    assert shares(1, H=128, Hkv=128, ordered=True, **rows) == (2, 2, 2)
    assert shares(1, H=129, Hkv=129, ordered=True, **rows) == (2, 1, 1)
    assert shares(1, H=257, Hkv=257, ordered=True, **rows) == (1, 1, 1)


def test_few_pairs_whatever_the_batch():
    for nb in (1, 1000):
        assert shares(nb, 64, 64, 12, 12, 64) == shares(nb, 1, 64, 12, 3, 128) == (2, 2, 2)
    assert shares(1000, 65, 64, 12, 12, 64) == shares(1000, 64, 65, 12, 12, 64) == (1, 1, 1)


def test_f32():
    rows = dict(Sq=200, Sk=200, dh=64, bf16=False)            # four blocks of 64 rows a head
    assert shares(1, H=63, Hkv=63, **rows) == (2, 2, 2)
    assert shares(1, H=64, Hkv=64, **rows) == (1, 2, 2)
    assert shares(1, H=128, Hkv=64, **rows) == (1, 1, 2)
    assert shares(1, H=128, Hkv=128, **rows) == (1, 1, 1)


def test_counts_that_pass_32_bits():
    assert shares(1 << 14, Sq=1 << 14, Sk=1 << 14, H=1 << 12, Hkv=1 << 12, dh=64) == (1, 1, 1)
