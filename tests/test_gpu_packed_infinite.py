"""Attention over packed prompts with infinite keys and queries: what the softmax gives.  A score of -inf
has the weight 0, however many of a row's first keys have one; one of +inf or NaN, or nothing but -inf, makes the row NaN.
The bound of finite rows is that of test_gpu_packed.py."""
import numpy as np
import pytest

import kv8_ref as ref
import test_gpu_packed as packed

pytestmark = pytest.mark.gpu


def _expect(q, k, v, at):
    """(o, bound): in float64, NaN where the softmax has no value."""
    T, H, dh = q.shape
    G = H // k.shape[1]
    o, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for a, b in zip(at, at[1:]):
        for h in range(H):
            qq, kk, vv = (x.astype(np.float64) for x in (q[a:b, h], k[a:b, h // G], v[a:b, h // G]))
            with np.errstate(all="ignore"):
                s = np.stack([(kk * row).sum(1) for row in qq]) / np.sqrt(dh)
            for t in range(b - a):
                x, n = s[t, :t + 1], t + 1
                if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
                    continue
                w = np.exp(x - x.max())
                w /= w.sum()
                seen = x > -np.inf
                off = (np.abs(qq[t]) * np.abs(kk[:n][seen])).sum(1).max() / np.sqrt(dh) * (dh + 4) * 2.0 ** -24
                o[a + t, h] = w @ vv[:n]
                tol[a + t, h] = (w @ np.abs(vv[:n])) * (2 * 2.0 ** -8 + 2 * off + (n + 64) * 2.0 ** -24) + np.abs(o[a + t, h]) * 2.0 ** -8 + 1e-37
    return o, tol


def _check(q, k, v, at):
    o = packed._run(q, k, v, at)
    want, tol = _expect(q, k, v, at)
    none = np.isnan(want)
    assert np.isnan(o[none]).all()
    assert np.all(np.abs(o - want)[~none] <= tol[~none])
    return none


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("keys", [1, 2, 31, 32, 63, 64, 65, 128, 130, 200])
def test_first_keys_infinite(dh, keys):
    """A prompt's first keys have an infinity in one dim: by its sign and the query's, scores of -inf or +inf."""
    H, Hkv = 2, 1
    at = [0, 40, 300]
    q, k, v = packed._inputs(("inf", dh, keys), at[-1], H, Hkv, dh)
    k[at[1]:at[1] + keys, 0, 5] = -np.inf
    q[:, 0, 5] = np.abs(q[:, 0, 5]) + 1
    q[:, 1, 5] = np.where(np.arange(at[-1]) % 3, q[:, 0, 5], -1)
    none = _check(q, k, v, at)
    rows = at[1] + keys
    assert none[at[1]:rows].all() and not none[rows:, 0].any() and not none[:at[1]].any()
    assert np.array_equal(none[rows:, 1, 0], np.arange(rows, at[-1]) % 3 == 0)


@pytest.mark.parametrize("dh", [64, 128])
def test_single_keys_and_queries(dh):
    H, Hkv = 4, 2
    at = [0, 70, 330]
    q, k, v = packed._inputs(("infs", dh), at[-1], H, Hkv, dh)
    for i, where in enumerate((0, 31, 32, 69, 70, 100, 133, 134, 197, 198, 300, 329)):
        kk = k.copy()
        kk[where, 1, 3] = [np.inf, -np.inf][i % 2]
        none = _check(q, kk, v, at)
        assert not none[:, :2].any()
    qq = q.copy()
    qq[150, 1, 0], qq[3, 2, 1], qq[250, 3, 2] = np.inf, -np.inf, np.inf
    none = _check(qq, k, v, at)
    assert none[150, 1].all() and none[3, 2].all() and none[250, 3].all() and none.sum() == 3 * dh


def test_products_past_fp32():
    """Finite keys whose products with the query leave fp32 below, over whole tiles: no weight, as in the limit."""
    T, H, dh = 300, 1, 64
    q, k, v = packed._inputs(("far",), T, H, H, dh)
    k[:130, 0, 0], q[:, 0, 0] = ref.bf16(np.full(130, -3e38)), 8.0
    o = packed._run(q, k, v, [0, T])
    want, tol = _expect(q[130:], k[130:], v[130:], [0, T - 130])
    assert np.all(np.abs(o[130:] - want) <= tol)
