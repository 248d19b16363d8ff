"""The size of the 4-bit attention's scratch, on the CPU."""
import random

import pytest

from paper_2608_14586_amd import binding as vb


@pytest.mark.parametrize("B,Lq,H,Hkv,dh,window,sinks", [
    (8, 1, 32, 8, 128, 0, 0), (3, 4, 32, 32, 128, 0, 0), (1, 1, 32, 32, 128, 0, 0), (1, 1, 8, 1, 64, 0, 0),
    (4, 1, 14, 2, 64, 0, 0), (16, 3, 32, 8, 128, 1024, 4), (2, 70, 12, 3, 64, 5000, 300), (300, 1, 40, 8, 128, 0, 0)])
def test_never_falls_with_the_length(B, Lq, H, Hkv, dh, window, sinks):
    """One allocation for the longest call serves a program whose max_len grows."""
    last = 0
    for n in list(range(0, 9000, 16)) + list(range(9000, 200000, 1000)) + [1 << 20, 1 << 24]:
        size = vb.vla_op_attention_kv4_scratch(B, Lq, H, Hkv, dh, n, window, sinks)
        assert size >= last, n
        last = size


def test_never_falls_with_the_length_drawn():
    rng = random.Random(5)
    for _ in range(300):
        Hkv = rng.choice([1, 2, 3, 4, 8, 32])
        a = (rng.randint(1, 64), rng.choice([1, 1, 2, 5, 40]), Hkv * rng.randint(1, 12), Hkv, rng.choice([64, 128]))
        w = (rng.choice([0, 0, rng.randint(1, 5000)]), rng.randint(0, 200))
        lens = sorted(rng.randint(0, 1 << rng.randint(1, 20)) for _ in range(40))
        sizes = [vb.vla_op_attention_kv4_scratch(*a, n, *w) for n in lens]
        assert sizes == sorted(sizes), (a, w)


def test_is_small():
    """At most 16 rows of dh + 2 numbers for 8192 workgroups, and for one more of each tile."""
    for B, Lq, H, Hkv in ((1, 1, 32, 8), (64, 1, 32, 8), (16, 8, 64, 4), (1, 64, 16, 16)):
        assert vb.vla_op_attention_kv4_scratch(B, Lq, H, Hkv, 128, 1 << 24) <= (8192 + B * Lq * H) * 16 * 130 * 4
