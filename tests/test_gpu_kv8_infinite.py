"""Attention over the 8-bit cache: queries that are not finite, and scores at the lower end of fp32."""
import numpy as np
import pytest

import kv8_ref as ref
import test_gpu_kv8 as kv8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,H,Hkv,Lq,window,sinks", [(1, 2, 2, 1, 0, 0), (1, 4, 1, 3, 0, 0), (40, 4, 2, 2, 0, 0), (700, 8, 1, 1, 0, 0),
                                                     (5000, 4, 1, 5, 0, 0), (700, 4, 2, 3, 50, 3), (3000, 40, 1, 4, 0, 0)])
def test_queries_that_are_not_finite(dh, n, H, Hkv, Lq, window, sinks):
    """An infinity that meets keys of one sign makes every score of its row -inf, or +inf: NaN either way, as for
    NaN itself; other rows keep their bits, and a row without a key is zeros."""
    L_cap = (n + 31) // 32 * 32
    k, v = kv8._kv(("notfinite", n, dh), 1, n, Hkv, dh)
    k[..., 3] = -np.abs(k[..., 3]) - 0.5
    q = ref.normal(("notfiniteq", n, dh, Lq), (1, Lq, H, dh))
    cache, _ = kv8._filled(k, v, L_cap, [n])
    base = kv8._attend(q, cache, L_cap, Hkv, [n], n, window, sinks)
    assert np.isfinite(base).all()
    for bad in (np.inf, -np.inf, np.nan):
        for i, h in ((Lq - 1, 0), (0, H - 1)):
            x = q.copy()
            x[0, i, h, 3] = bad
            o = kv8._attend(x, cache, L_cap, Hkv, [n], n, window, sinks)
            assert np.isnan(o[0, i, h]).all() if n - Lq + i >= 0 else not o[0, i, h].any(), (bad, i, h)
            o[0, i, h] = base[0, i, h]
            assert np.array_equal(o, base)


@pytest.mark.parametrize("n", [1, 33, 3000])
def test_scores_at_the_end_of_fp32(n):
    """All scores are -3.32e38 (in log2): weights are alike, and the result is the values' mean.  It is off by its n
    roundings in fp32, the last one to bf16 (2^-8), and of the sum of |v| by 2^-24 for each addition."""
    dh, L_cap = 64, (n + 31) // 32 * 32
    k, v = np.zeros((1, n, 1, dh), np.float32), ref.normal(("end", n), (1, n, 1, dh))
    k[..., 0] = -352 * 2.0 ** 118  # a code times a power of two
    q = np.zeros((1, 1, 2, dh), np.float32)
    q[..., 0] = 15.75
    assert -3.4e38 < 15.75 * float(k[0, 0, 0, 0]) / 8 * np.log2(np.e) < -3e38
    cache, held = kv8._filled(k, v, L_cap, [n])
    o = kv8._attend(q, cache, L_cap, 1, [n], n)
    x = held[1][0][:n, 0]
    want = x.mean(0)
    assert np.all(np.abs(o[0, 0] - want) <= np.abs(want) * 2.0 ** -8 + np.abs(x).mean(0) * (n + 64) * 2.0 ** -24 + 1e-37)
