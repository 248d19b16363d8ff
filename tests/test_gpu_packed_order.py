"""Attention over packed prompts where all workgroups run at once and take tiles in pairs (257 to 512 tiles and
heads), and on both sides of that range: against float64, and to the last bit what each prompt gives alone.
The bound is that of test_gpu_packed.py."""
import numpy as np
import pytest

import test_gpu_packed as packed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,dh,lens,tiles", [
    (1, 1, 64, [512] * 62 + [1100], 257),           # one more than there are CUs
    (32, 8, 64, [511, 300, 8], 256),                # the last in plain order
    (14, 2, 64, [701, 64, 1, 333, 128, 417, 95, 256, 29], 280),
    (14, 2, 128, [700] * 3 + [500], 308),
    (32, 32, 128, [1000, 100], 288),
    (5, 1, 128, [50] * 40 + [1500], 260),           # no multiple of the heads is 256
    (14, 2, 64, [100] * 36, 504),                   # one tile a prompt
    (7, 7, 64, [90] * 40 + [4111], 511),
    (32, 8, 128, [2048], 512),                      # two tiles for every CU
    (32, 4, 64, [1, 127, 128, 129, 255, 257, 600], 480),
    (19, 1, 64, [300] * 8 + [257], 513),            # plain order again
    (14, 2, 128, [65] * 30 + [1700], 616),
    (32, 8, 64, [129] * 20, 1280),
])
@pytest.mark.parametrize("pad", [0, 700])
def test_tiles_in_every_order(H, Hkv, dh, lens, tiles, pad):
    at = packed._offsets(lens, pad // 7)
    assert sum((n + 127) // 128 for n in lens) * H == tiles
    q, k, v = packed._inputs(("order", H, dh, len(lens)), at[-1] + pad, H, Hkv, dh)
    o = packed._run(q, k, v, at)
    packed._check(o, q, k, v, at)
    for a, b in list(zip(at, at[1:]))[-4:]:
        assert np.array_equal(o[a:b], packed._run(q[a:b], k[a:b], v[a:b], [0, b - a])), (a, b)
