"""The largest bf16 numbers in the 8-bit cache: which of them load as infinity, and what attention makes of them."""
import numpy as np
import pytest

import kv8_ref as ref
import test_gpu_kv8 as kv8

pytestmark = pytest.mark.gpu


def test_which_finite_values_load_as_infinity():
    """Those from 248 2^120 on, the middle between 240 2^120 and 2^128; each in a block of its own, and all in one block of 32."""
    bits = np.concatenate([np.arange(0x7f00, 0x7f80), np.arange(0xff00, 0xff80)]).astype(np.uint32) << 16
    x = bits.view(np.float32)
    assert np.isfinite(x).all()
    big = np.abs(x.astype(np.float64)) >= 248 * 2.0 ** 120
    assert big.sum() == 2 * 8
    dh, n = 64, len(x)
    alone = np.zeros((1, 32 * n, 1, dh), np.float32)
    alone[0, ::32, 0, 5] = x
    together = np.zeros((1, n, 1, dh), np.float32)
    together[0, :, 0, 5] = x
    for rows, step in ((alone, 32), (together, 1)):
        L = rows.shape[1]
        cache = kv8._cache(1, 1, L, dh)
        kv8._vb().vla_op_kv8_store(ref.to_dev(rows), ref.to_dev(rows), None, None, cache, L)
        for y in kv8._load(cache, L, 1, L, 1, dh):
            y = y[0, ::step, 0, 5]
            assert np.array_equal(np.isinf(y), big) and np.array_equal(np.sign(y), np.sign(x))
            # the others by half a step of 4 significant bits at most
            assert np.all(np.abs(y - x.astype(np.float64))[~big] <= 2.0 ** -4 * np.abs(x.astype(np.float64))[~big])


def test_attention_over_them():
    """Two keys of equal weight: the mean of 2^128 and of a smaller value is a number, and is right to its roundings."""
    dh = 64
    k, q = np.zeros((1, 2, 1, dh), np.float32), ref.normal(("largest",), (1, 1, 2, dh))
    v = np.zeros((1, 2, 1, dh), np.float32)
    v[0, 0], v[0, 1, 0, ::2] = 3.3895314e38, -3.3895314e38 / 4
    assert np.array_equal(ref.bf16(v[0, 0]), v[0, 0])
    cache, held = kv8._filled(k, v, 32, [2])
    assert (held[1][0][0] == 2.0 ** 128).all()
    o = kv8._attend(q, cache, 32, 1, [2], 2)
    want = held[1][0][:2, 0].mean(0)
    assert np.isfinite(o).all() and np.all(np.abs(o[0, 0] - want) <= np.abs(want) * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -20))
