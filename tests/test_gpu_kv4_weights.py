"""Attention over the 4-bit cache where keys weigh very differently: large values
that a query does not see or gives no weight, values of all sizes, and every way
of splitting the work.  The bound is a sum over the keys that a query sees, each
by its weight: what has no weight allows no error."""
import numpy as np
import pytest

import w4kv4_ref as ref
from test_gpu_kv4 import _attend, _cache, _kv

pytestmark = pytest.mark.gpu


def attention_and_bound(q, k, v, length, window, sinks, steps=None):
    """o[Lq][H][dh] of one sequence in float64 over the cached values, and how far
    a result may be off.  Per query, head and group of 32 dims, with p the softmax
    weights, s and m a key's step and minimum in the cache:
      - the result's rounding to bf16: 2^-8 of it;
      - the rounding of p s to fp16, half a step or 2^-11 of it, times a code counted
        from the middle: 2^-11 * 7.5 sum p s;
      - scores: a group's sum of (16 + c) q starts from -16 sum q, 47 sum |q| in all,
        and takes m sum q: 34 fp32 roundings for the sums and two a group where the
        groups are joined, each at most 2^-24 of sum_g (47 s + |m|) sum |q|; then two
        of the score itself (2^-23), and the exponential (2^-21).  A weight's relative
        error e moves the result by p e (|v| + |o|);
      - sums over keys in fp32: of p s (b + c) and p s (b + 7.5), each at most 271 p s, one
        rounding a block and 32 in it, and of p m, two a block; 100 more to join
        waves and splits.  `steps`: how many blocks a wave takes at most."""
    Lq, H, dh = q.shape
    Hkv = k.shape[1]
    G, NG = H // Hkv, dh // 32
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    steps = -(-length // 32) if steps is None else steps
    for h in range(Hkv):
        (ck, sk, mk), (cv, sv, mv) = ref.quantise(k[:length, h]), ref.quantise(v[:length, h])
        kk, vv = (mk + sk * ck).reshape(length, dh), (mv + sv * cv).reshape(length, dh)
        mag = np.repeat((np.abs(mv) + 15 * sv)[..., 0], 32, -1)
        for i in range(Lq):
            see = ref.visible(length - Lq + i, length, window, sinks)
            if not see.any():
                continue
            at = slice(None) if see.all() else see
            x = q[i, h * G:(h + 1) * G]
            w = x @ kk[at].T / np.sqrt(dh)
            p = np.exp(w - w.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            y = p @ vv[at]
            aq = np.abs(x).reshape(G, NG, 32).sum(-1)
            err = 2.0 ** -24 * (34 + 2 * NG) / np.sqrt(dh) * (aq @ (47 * sk + np.abs(mk))[at][..., 0].T)
            err = 1.1 * (err + 2.0 ** -23 * np.abs(w)) + 2.0 ** -21
            assert (err < 0.1).all()  # e^x - 1 <= 1.1 x
            ps = np.repeat(p @ sv[at][..., 0], 32, -1)
            e = (p * err) @ np.abs(vv[at]) + (p * err).sum(-1, keepdims=True) * np.abs(y)
            e += 2.0 ** -11 * 7.5 * ps
            e += 2.0 ** -24 * ((steps + 132) * 542 * ps + (2 * steps + 132) * (p @ mag[at]))
            o[i, h * G:(h + 1) * G] = y
            bound[i, h * G:(h + 1) * G] = 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -7) * e + 2.0 ** -126
    return o, bound


def _check(got, q, k, v, lens, window=0, sinks=0, steps=None):
    for b, n in enumerate(lens):
        want, bound = attention_and_bound(q[b], k[b], v[b], n, window, sinks, steps)
        over = np.abs(got[b] - want) / np.maximum(bound, 1e-300)
        assert (over <= 1).all(), (b, np.unravel_index(np.argmax(over), over.shape), over.max())


def _stored(k, v, lens, L_cap):
    from paper_2608_14586_amd import binding as vb
    import torch
    cache = _cache(k.shape[0], k.shape[2], L_cap, k.shape[3], 255)  # unwritten rows: NaN
    count = torch.tensor(lens, dtype=torch.int32, device="cuda")
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, count, cache, L_cap)
    return cache


@pytest.mark.parametrize("power", [10, 20, 24, 28, 34, 60, 110])
@pytest.mark.parametrize("dh,n,window,sinks", [(64, 32, 0, 0), (128, 45, 0, 0), (64, 300, 0, 0), (128, 700, 90, 3)])
def test_values_that_a_query_does_not_see(power, dh, n, window, sinks):
    _unseen(power, 1, 3, 2, 2, dh, n, window, sinks)  # a head's three queries share a tile


@pytest.mark.parametrize("power", [20, 34])
@pytest.mark.parametrize("B,Lq,H,Hkv,dh,n", [(13, 11, 7, 1, 64, 420), (13, 11, 7, 1, 128, 3000), (3, 19, 36, 3, 64, 900)])
def test_values_that_a_query_of_a_large_tile_does_not_see(power, B, Lq, H, Hkv, dh, n):
    _unseen(power, B, Lq, H, Hkv, dh, n, 0, 0)


def _unseen(power, B, Lq, H, Hkv, dh, n, window, sinks):
    """The last of several tokens, and with a window those between the first
    tokens and the last query's window, have values 2^power times the others'.  Queries
    that do not see them: the result without them, to the last bit, and right."""
    k, v = _kv(("unseen", dh, n), B, n, Hkv, dh)
    q = ref.normal(("unseenq", dh, n), (B, Lq, H, dh))
    big = v.copy()
    big[:, -1] = ref.bf16(big[:, -1] * 2.0 ** power)  # the last query alone sees it
    if window:  # the first query alone sees this one
        big[:, n - Lq - window + 1] = ref.bf16(big[:, n - Lq - window + 1] * 2.0 ** power)
    cap = (n + 31) // 32 * 32
    a = _attend(ref.to_dev(q), _stored(k, v, [n] * B, cap), cap, Hkv, [n] * B, n, window, sinks)
    b = _attend(ref.to_dev(q), _stored(k, big, [n] * B, cap), cap, Hkv, [n] * B, n, window, sinks)
    free = slice(1 if window else 0, Lq - 1)
    assert np.array_equal(a[:, free], b[:, free])
    _check(b, q, k, big, [n] * B, window, sinks)


@pytest.mark.parametrize("power", [10, 20, 24, 28, 34, 50])
@pytest.mark.parametrize("dh,H,Hkv,Lq,n", [(64, 2, 2, 1, 32), (128, 4, 1, 1, 1024), (64, 14, 2, 1, 500), (64, 7, 1, 11, 130),
                                           (64, 7, 1, 11, 420), (128, 7, 1, 11, 3000)])
def test_values_without_weight(power, dh, H, Hkv, Lq, n):
    """One early token that every query sees has a score about 60 below the others
    and values 2^power times theirs, less than its weight of 2^-85 takes away."""
    B = 13 if Lq > 1 else 1
    k, v = _kv(("weightless", dh, n), B, n, Hkv, dh)
    q = ref.normal(("weightlessq", dh, n), (B, Lq, H, dh))
    k[..., 0], q[..., 0] = 0.0, 8.0  # one channel is this token's alone: a score of -60 more
    at = 5
    k[:, at, :, 0] = ref.bf16(-60.0 * np.sqrt(dh) / 8.0)
    v[:, at] = ref.bf16(v[:, at] * 2.0 ** power)
    cap = (n + 31) // 32 * 32
    got = _attend(ref.to_dev(q), _stored(k, v, [n] * B, cap), cap, Hkv, [n] * B, n)
    _check(got, q, k, v, [n] * B)


@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("dh,n", [(64, 640), (128, 900)])
def test_values_and_scores_that_run_apart(falling, dh, n):
    """Scores that rise from token to token by 200 in all while the values fall by
    2^150, and the other way around: the range of what was seen before has to give way."""
    B, H, Hkv = 1, 4, 2
    k, v = _kv(("apart", dh, n), B, n, Hkv, dh)
    q = ref.normal(("apartq", dh, n), (B, 1, H, dh))
    q[..., 0] = 8.0
    t = np.arange(n) / (n - 1.0)
    t = 1 - t if falling else t
    k[..., 0] = ref.bf16((t * 200.0 * np.sqrt(dh) / 8.0)[None, :, None])
    v = ref.bf16(v * (2.0 ** np.rint(75 - 150 * t))[None, :, None, None])
    cap = (n + 31) // 32 * 32
    got = _attend(ref.to_dev(q), _stored(k, v, [n], cap), cap, Hkv, [n], n)
    _check(got, q, k, v, [n])


@pytest.mark.parametrize("B,Lq,H,Hkv,dh,n", [(13, 11, 7, 1, 64, 129), (13, 11, 7, 1, 64, 420), (3, 19, 36, 3, 128, 900)])
def test_a_query_beside_one_that_is_not_finite(B, Lq, H, Hkv, dh, n):
    """Every other query's result is the same, to the last bit."""
    k, v = _kv(("besidenan",), B, n, Hkv, dh)
    cap = (n + 31) // 32 * 32
    cache = _stored(k, v, [n] * B, cap)
    q = ref.normal(("besidenanq",), (B, Lq, H, dh))
    want = _attend(ref.to_dev(q), cache, cap, Hkv, [n] * B, n)
    for bad in (np.nan, np.inf, 1e30):
        x = q.copy()
        x[:, 4, 3, 5] = ref.bf16(bad)
        got = _attend(ref.to_dev(x), cache, cap, Hkv, [n] * B, n)
        assert np.isfinite(want).all() and (bad == 1e30 or np.isnan(got[:, 4, 3]).all())
        got[:, 4, 3] = want[:, 4, 3]
        assert np.array_equal(got, want)


@pytest.mark.parametrize("n", [64, 70])
def test_values_that_are_not_finite(n):
    """A key that a query sees, of a weight that is 0 in fp32, with a value that is
    not finite: NaN in that group of 32 dims, whether the key's block is seen whole or
    in part, and in no other group; a query that does not see it is as without it."""
    B, Lq, H, Hkv, dh = 1, 2, 4, 2, 128
    for at in (3, n - 1):
        k, v = _kv(("notfinite", n), B, n, Hkv, dh)
        q = ref.normal(("notfiniteq", n), (B, Lq, H, dh))
        k[..., 0], q[..., 0] = 0.0, 8.0
        k[:, at, :, 0] = ref.bf16(-300.0 * np.sqrt(dh) / 8.0)
        bad = v.copy()
        bad[:, at, :, 40] = np.inf
        cap = (n + 31) // 32 * 32
        a = _attend(ref.to_dev(q), _stored(k, v, [n], cap), cap, Hkv, [n], n)
        b = _attend(ref.to_dev(q), _stored(k, bad, [n], cap), cap, Hkv, [n], n)
        sees = [0, 1] if at == 3 else [1]
        assert np.isnan(b[0, sees][..., 32:64]).all()
        b[0, sees, :, 32:64] = a[0, sees, :, 32:64]
        assert np.array_equal(a, b)


@pytest.mark.parametrize("n", [1, 2, 40])
def test_the_largest_values(n):
    """Values whose steps reach 2^124: the weighted sums stay in fp32."""
    B, H, Hkv, dh = 1, 4, 2, 64
    k, v = _kv(("largest", n), B, n, Hkv, dh)
    v = ref.bf16(np.sign(v) * 2.0 ** 127)
    q = ref.normal(("largestq", n), (B, 1, H, dh))
    cap = (n + 31) // 32 * 32
    got = _attend(ref.to_dev(q), _stored(k, v, [n], cap), cap, Hkv, [n], n)
    assert np.isfinite(got).all()
    _check(got, q, k, v, [n])


@pytest.mark.parametrize("dh", [64, 128])
def test_the_largest_value_behind_others(dh):
    """A key whose score is up to 2^8 above those seen before it, so that it moves no
    maximum, with values of 2^127: its weight is nearly 1 there, and 256 steps
    of it would not be finite."""
    B, H, Hkv, n = 1, 8, 1, 600  # three blocks of 32 for each of eight waves
    k, v = _kv(("behind", dh), B, n, Hkv, dh)
    q = ref.normal(("behindq", dh), (B, 1, H, dh), 0.1)
    k[..., 0], q[..., 0] = 0.0, 8.0
    k[:, 301, :, 0] = ref.bf16(5.0 * np.sqrt(dh) / 8.0)
    v[:, 301] = ref.bf16(np.sign(v[:, 301]) * 2.0 ** 127)
    got = _attend(ref.to_dev(q), _stored(k, v, [n], 608), 608, Hkv, [n], n)
    assert np.isfinite(got).all()
    _check(got, q, k, v, [n])


@pytest.mark.parametrize("Lq,n", [(1, 1), (3, 3), (1, 2), (1, 40)])
@pytest.mark.parametrize("dh", [64, 128])
def test_rounding_of_the_weights(Lq, n, dh):
    """Values of 0 in groups of a minimum -15 a and step a = 1, so that the result is 0 and
    nothing but the rounding of p s shows: at most 2^-11 * 7.5 sum p s, the codes
    counted from their middle, and less than 2^-10 from the sums in fp32 (at most
    279 sum p s, 44 roundings of 2^-24)."""
    B, H, Hkv = 1, 64, 1
    k, _ = _kv(("rounding", dh, n), B, n, Hkv, dh)
    q = ref.normal(("roundingq", dh, n), (B, Lq, H, dh))
    v = np.zeros((B, n, Hkv, dh))
    v[..., ::32] = -15.0
    got = _attend(ref.to_dev(q), _stored(k, v, [n], 64), 64, Hkv, [n], n)
    got = got.reshape(Lq, H, dh // 32, 32)
    assert (np.abs(got[..., 0] + 15) <= 2.0 ** -8 * 15).all()
    assert (np.abs(got[..., 1:]) <= (1 + 2.0 ** -8) * (2.0 ** -11 * 7.5 + 2.0 ** -10)).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("bits", [16, 19, 22, 25, 28, 31])
def test_many_small_weights(bits, dh):
    """One key, and 4000 of weights 2^-bits of its: their p s are subnormal as fp16, or
    nothing, and what the codes' offset of up to 256 makes of them is taken off to
    the last bit.  The one key's values are 0, which leaves nothing else to see."""
    B, H, Hkv, n = 1, 8, 1, 4000
    k, v = _kv(("small", dh), B, n, Hkv, dh)
    q = ref.normal(("smallq", dh), (B, 1, H, dh), 0.02)
    k[..., 0], q[..., 0] = 0.0, 8.0
    k[:, 0, :, 0] = ref.bf16(bits * np.log(2) * np.sqrt(dh) / 8.0)
    v[:, 0] = np.where(np.arange(dh) % 32 == 0, -15.0, 0.0)
    got = _attend(ref.to_dev(q), _stored(k, v, [n], n), n, Hkv, [n], n)
    _check(got, q, k, v, [n], steps=17)


# Sizes at which the call takes 4, 8 and 16 queries a tile, each with 4 and 8 waves,
# one split, several, and more than the 64 that are joined at a time; no number of
# query rows is a multiple of the tile's.  The last column: blocks a wave takes at most.
SPLITS = [
    (1, 1, 1, 1, 33, 1), (1, 1, 1, 1, 1500, 1), (1, 1, 1, 1, 129, 1), (1, 1, 1, 1, 9000, 1), (1, 1, 1, 1, 40000, 2),
    (1, 11, 3, 1, 4000, 2), (3, 19, 36, 3, 33, 1), (1, 11, 12, 1, 2000, 2), (1, 19, 5, 1, 1500, 1), (1, 19, 5, 1, 3017, 2),
    (13, 11, 21, 3, 33, 1), (2, 19, 9, 3, 2000, 2), (13, 11, 7, 1, 420, 2), (1, 11, 12, 1, 6000, 2), (1, 19, 1, 1, 40000, 2),
    (8, 19, 96, 8, 33, 1), (13, 11, 7, 1, 3000, 4), (3, 19, 36, 3, 900, 4), (2, 19, 9, 3, 9000, 4), (1, 19, 1, 1, 80000, 4),
    (4, 8, 32, 4, 1100, 5), (13, 11, 7, 1, 129, 2), (3, 19, 36, 3, 129, 2), (1, 11, 12, 1, 4000, 3),
]
LONGEST = (1, 5, 5, 1, 200000, 7)  # 16 queries a tile and more than 64 splits


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("case", range(len(SPLITS)))
def test_every_way_to_split(case, dh):
    _split(case, dh, *SPLITS[case])


def test_many_splits_of_large_tiles():
    _split("longest", 64, *LONGEST)


def _split(case, dh, B, Lq, H, Hkv, n, steps):
    lens = [n - (b * n) // (2 * B) for b in range(B)]
    k, v = _kv(("splits", case, dh), B, n, Hkv, dh)
    # no two parts of the sequence have the same mean: none can be left out or taken twice
    v = ref.bf16(v + 2 * np.cos(np.pi * np.arange(n) / n)[None, :, None, None])
    q = ref.normal(("splitsq", case, dh), (B, Lq, H, dh))
    cap = (n + 31) // 32 * 32
    got = _attend(ref.to_dev(q), _stored(k, v, lens, cap), cap, Hkv, lens, n)
    _check(got, q, k, v, lens, steps=steps + 1)


@pytest.mark.parametrize("B,Lq,H,Hkv,n,window,sinks", [(16, 3, 32, 8, 1500, 1024, 4), (5, 7, 12, 3, 600, 50, 40), (3, 13, 8, 2, 333, 1, 0)])
def test_windows_of_several_queries(B, Lq, H, Hkv, n, window, sinks):
    dh = 64
    lens = [max(1, n - 101 * b) for b in range(B)]
    k, v = _kv(("windows", B, Lq), B, n, Hkv, dh)
    q = ref.normal(("windowsq", B, Lq), (B, Lq, H, dh))
    cap = (n + 31) // 32 * 32
    got = _attend(ref.to_dev(q), _stored(k, v, lens, cap), cap, Hkv, lens, n, window, sinks)
    _check(got, q, k, v, lens, window, sinks)


@pytest.mark.parametrize("B,Lq,H,Hkv,dh,longest", [(8, 1, 32, 8, 128, 1000), (3, 4, 8, 8, 64, 2048)])
def test_one_scratch_for_a_growing_length(B, Lq, H, Hkv, dh, longest):
    """Scratch sized once, for the longest call, serves every shorter one."""
    import torch
    from paper_2608_14586_amd import binding as vb
    k, v = _kv(("growing", dh), B, longest, Hkv, dh)
    q = ref.normal(("growingq", dh), (B, Lq, H, dh))
    cache = _stored(k, v, [longest] * B, longest + 31 & ~31)
    scratch = torch.empty(vb.vla_op_attention_kv4_scratch(B, Lq, H, Hkv, dh, longest), dtype=torch.uint8, device="cuda")
    dq, o = ref.to_dev(q), torch.empty((B, Lq, H, dh), dtype=torch.bfloat16, device="cuda")
    for n in (Lq, 37, 130, 500, longest * 15 // 16, longest):
        scratch.fill_(255)
        lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
        vb.vla_op_attention_kv4(dq, cache, longest + 31 & ~31, Hkv, lens, o, n, 0, 0, scratch)
        _check(ref.from_dev(o), q, k, v, [n] * B)
