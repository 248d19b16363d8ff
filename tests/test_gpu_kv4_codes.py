"""The codes of the 4-bit cache where values of one group differ much in size: the
difference to the group's minimum is an fp32 number, and the code that divided by
the step, rounded once."""
import numpy as np
import pytest

import synth
import w4kv4_ref as ref
from test_gpu_kv4 import _cache, _load

pytestmark = pytest.mark.gpu


def _cached(x):
    """What rows x[..., dh] read back as, bf16 as float64."""
    g = x.reshape(x.shape[:-1] + (-1, 32))
    lo, hi = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
    f32 = lambda a: np.asarray(a, np.float32)  # noqa: E731
    s = ref.bf16((f32(hi - lo) * np.float32(1 / 15)).astype(np.float64))
    t = f32(g - lo).astype(np.float64)  # bf16 numbers: their difference is exact in 64 bits, and rounded once here
    return ref.bf16(lo + s * np.minimum(np.rint(t / s), 15)).reshape(x.shape)


def _check(x):
    from paper_2608_14586_amd import binding as vb
    B, L, H, dh = x.shape
    cap = (L + 31) // 32 * 32
    cache = _cache(B, H, cap, dh)
    vb.vla_op_kv4_store(ref.to_dev(x), ref.to_dev(-x), None, None, cache, cap)
    k, v = _load(cache, cap, B, L, H, dh)
    assert np.array_equal(k, _cached(x)) and np.array_equal(v, _cached(-x))


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -60, 2.0 ** 90])
def test_differences_that_round_onto_a_border(scale):
    """Minimums of -(k + 1/2) steps and values around 0, from far below to above what
    the difference's last bit holds."""
    small = np.concatenate([[0.0], *[[2.0 ** -p, -2.0 ** -p, 1.5 * 2.0 ** -p] for p in (16, 20, 21, 22, 23, 24, 25, 30, 60)]])
    x = np.zeros((1, 15, 1, 64))
    for k in range(15):
        for g in range(2):
            x[0, k, 0, 32 * g:32 * g + len(small)] = small * (1 + g / 4)
            x[0, k, 0, 32 * g + 30], x[0, k, 0, 32 * g + 31] = -(k + 0.5) * (1 + g / 4), (14.5 - k) * (1 + g / 4)
    assert np.array_equal(ref.bf16(x * scale), x * scale)
    assert _cached(x)[0, 2, 0, small.tolist().index(2.0 ** -30)] == -0.5  # code 2, as of 2.5 itself
    _check(x * scale)


@pytest.mark.parametrize("dh", [64, 128])
def test_values_of_many_sizes(dh):
    rng = np.random.default_rng(synth.seed_of("codes", dh))
    x = rng.normal(size=(2, 200, 3, dh)) * 2.0 ** rng.integers(-40, 3, (2, 200, 3, dh))
    steps = rng.integers(0, 31, x.shape) / 2.0  # and on the borders of a step of 1
    x[:, 100:] = np.where(rng.random(x[:, 100:].shape) < 0.5, x[:, 100:] * 2.0 ** -20, steps[:, 100:] - 7.5)
    x[:, 100:, :, ::32], x[:, 100:, :, 1::32] = -7.5, 7.5
    _check(ref.bf16(x))
