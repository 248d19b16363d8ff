"""Causal attention over packed prompts, against float64.

Weights are bf16 (2^-8 each) and their sum is of the rounded ones, so a result is off by
2 2^-8 of sum w |v| at most; scores are fp32 sums of dh exact products; sums over n keys
are fp32; the result is a bf16 (2^-8)."""
import numpy as np
import pytest

import kv8_ref as ref

pytestmark = pytest.mark.gpu


def _vb():
    from paper_2608_14586_amd import binding
    return binding


def _i32(*v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _offsets(lens, first=0):
    return [first] + [first + int(x) for x in np.cumsum(lens)]


def _reference(q, k, v, at):
    """(o, bound), NaN where no prompt has the row."""
    T, H, dh = q.shape
    G = H // k.shape[1]
    o, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for a, b in zip(at, at[1:]):
        a, b = min(max(a, 0), T), min(max(b, 0), T)
        n = b - a
        if n <= 0:
            continue
        sees = np.tril(np.ones((n, n), bool))
        for h in range(H):
            kk, vv = k[a:b, h // G].astype(np.float64), v[a:b, h // G].astype(np.float64)
            qq = q[a:b, h].astype(np.float64)
            s = np.where(sees, qq @ kk.T / np.sqrt(dh), -np.inf)
            off = np.where(sees, np.abs(qq) @ np.abs(kk).T, 0).max(1, keepdims=True) / np.sqrt(dh) * (dh + 4) * 2.0 ** -24
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            o[a:b, h] = w @ vv
            tol[a:b, h] = (w @ np.abs(vv)) * (2 * 2.0 ** -8 + 2 * off + (n + 64) * 2.0 ** -24) + np.abs(o[a:b, h]) * 2.0 ** -8 + 1e-37
    return o, tol


def _inputs(tag, T, H, Hkv, dh, std=1.0):
    return [ref.normal((n,) + tag, (T, h, dh), std) for n, h in (("q", H), ("k", Hkv), ("v", Hkv))]


def _run(q, k, v, at, fill=5.0):
    import torch
    dq, dk, dv = (ref.to_dev(x) for x in (q, k, v))
    o = torch.full(q.shape, fill, dtype=torch.bfloat16, device="cuda")
    _vb().vla_op_attention_packed(dq, dk, dv, _i32(*at), o)
    return ref.from_dev(o)


def _check(o, q, k, v, at, fill=5.0):
    r, tol = _reference(q, k, v, at)
    outside = np.isnan(r)
    assert np.all(o[outside] == fill)
    bad = np.abs(o - r)[~outside] / tol[~outside]
    assert np.all(bad <= 1), (at[:8], float(bad.max()) if bad.size else 0)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (8, 8), (14, 2), (32, 8), (5, 1)])
@pytest.mark.parametrize("lens", [[1], [2, 31, 32, 33], [63, 64, 65, 1, 1], [127, 128, 129], [0, 100, 0, 0, 200], [511, 300, 7]])
def test_packed(dh, H, Hkv, lens):
    at = _offsets(lens)
    q, k, v = _inputs((dh, H, str(lens)), at[-1], H, Hkv, dh)
    _check(_run(q, k, v, at), q, k, v, at)


@pytest.mark.parametrize("lens", [[4100], [2048, 1000, 3], [1300, 5, 2200]])
def test_long_prompts(lens):
    at = _offsets(lens)
    for H, Hkv, dh in ((3, 1, 128), (2, 2, 64)):
        q, k, v = _inputs(("long", dh, str(lens)), at[-1], H, Hkv, dh, 1.5)
        _check(_run(q, k, v, at), q, k, v, at)


@pytest.mark.parametrize("n", [64, 65, 200, 1000])
def test_many_prompts(n):
    lens = np.random.default_rng(n).integers(0, 40 if n > 100 else 150, n)
    at = _offsets(lens)
    q, k, v = _inputs(("many", n), at[-1], 2, 1, 64)
    _check(_run(q, k, v, at), q, k, v, at)


def test_rows_outside_and_cut_offsets():
    """Rows before the first prompt and behind the last stay; offsets outside the rows are cut."""
    T, H, Hkv, dh = 300, 4, 2, 64
    q, k, v = _inputs(("out",), T, H, Hkv, dh)
    for at in ([10, 100, 250], [-50, 20, 20, 90], [200, 299, 1000, 2000], [300, 300], [0, 0, 0], [500, 600], [-9, -3, 2 ** 31 - 1]):
        _check(_run(q, k, v, at), q, k, v, at)


def test_strides():
    """Rows of a fused projection, heads before tokens, and an output inside other memory."""
    import torch
    T, H, Hkv, dh = 333, 6, 2, 128
    q, k, v = _inputs(("strides",), T, H, Hkv, dh)
    at = [0, 77, 200, 333]
    rows = torch.full((T, H + 2 * Hkv + 1, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:-1] = ref.to_dev(q), ref.to_dev(k), ref.to_dev(v)
    whole = torch.full((T, 2 * H, dh + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    o = whole[:, ::2, :dh]
    _vb().vla_op_attention_packed(rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:-1], _i32(*at), o)
    _check(ref.from_dev(o), q, k, v, at)
    assert bool((whole[:, 1::2] == 5).all()) and bool((whole[:, :, dh:] == 5).all())
    turned = [ref.to_dev(x).transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    o = torch.full((T, H, dh), 5.0, dtype=torch.bfloat16, device="cuda")
    _vb().vla_op_attention_packed(*turned, _i32(*at), o)
    _check(ref.from_dev(o), q, k, v, at)
    one = k[:, :1]
    wide = ref.to_dev(one).expand(T, Hkv, dh)  # a head stride of 0
    _vb().vla_op_attention_packed(turned[0], wide, turned[2], _i32(*at), o)
    _check(ref.from_dev(o), q, np.repeat(one, Hkv, 1), v, at)


@pytest.mark.parametrize("dh", [64, 128])
def test_values_that_are_not_finite(dh):
    """A key or value that is not finite reaches the rows behind it in its own prompt and no others; neither do rows outside."""
    H, Hkv = 4, 2
    at = [0, 70, 400, 460]
    T = 500
    q, k, v = _inputs(("nan", dh), T, H, Hkv, dh)
    k[460:], v[460:], q[460:] = np.nan, np.inf, np.nan
    base = _run(q, k, v, at)
    _check(base, q, k, v, at)
    for where in (0, 5, 31, 32, 40, 63, 64, 69, 70, 100, 133, 134, 197, 198, 300, 399, 400, 459):
        for part in ("k", "v"):
            kk, vv = k.copy(), v.copy()
            (kk if part == "k" else vv)[where, 1, 3] = [np.nan, np.inf, -np.inf][where % 3]
            o = _run(q, kk, vv, at)
            end = [b for b in at if b > where][0]
            hit = ~np.isfinite(o[:, 2:])  # the heads of KV head 1
            assert np.array_equal(o[:, :2], base[:, :2])
            sees = np.zeros(T, bool)
            sees[where:end] = True
            if part == "v":
                assert hit[sees, :, 3].all() and not np.delete(hit, 3, 2).any() and not hit[~sees].any(), where
                keep = ~hit
                assert np.array_equal(np.delete(o[:, 2:], 3, 2), np.delete(base[:, 2:], 3, 2)) and np.array_equal(o[:, 2:][keep], base[:, 2:][keep])
            else:
                if np.isnan(kk[where, 1, 3]):
                    assert hit[sees].all()
                assert not hit[~sees].any() and np.array_equal(o[~sees], base[~sees]), where
    qq = q.copy()
    qq[150, 1, 0] = np.nan
    o = _run(qq, k, v, at)
    assert np.isnan(o[150, 1]).all()
    o[150, 1] = base[150, 1]
    assert np.array_equal(o, base)


def test_large_scores():
    """Scores hundreds apart: the maximum moves tile by tile, and one key takes all the weight."""
    T, H, dh = 700, 2, 64
    q, k, v = _inputs(("peak",), T, H, H, dh)
    k = ref.bf16(k * 0.01)
    k[:, 0, 0], k[:, 1, 0] = ref.bf16(np.linspace(-400, 400, T)), ref.bf16(np.linspace(400, -400, T))
    q[..., 0] = 8
    _check(_run(q, k, v, [0, T]), q, k, v, [0, T])


def test_a_prompt_has_the_same_bits_alone():
    H, Hkv, dh = 8, 2, 128
    at = [0, 300, 301, 900]
    q, k, v = _inputs(("alone",), 900, H, Hkv, dh)
    o = _run(q, k, v, at)
    assert np.array_equal(o, _run(q, k, v, at))
    for a, b in zip(at, at[1:]):
        assert np.array_equal(o[a:b], _run(q[a:b], k[a:b], v[a:b], [0, b - a]))


def test_graph_with_other_offsets():
    """Captured once, replayed with other offsets and rows; on a stream of its own."""
    import torch
    T, H, Hkv, dh = 512, 4, 2, 64
    dq, dk, dv = (torch.empty((T, h, dh), dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv))
    o = torch.empty((T, H, dh), dtype=torch.bfloat16, device="cuda")
    off = _i32(0, 0, 0, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _vb().vla_op_attention_packed(dq, dk, dv, off, o)
    for i, at in enumerate(([0, 100, 300, 512], [0, 511, 511, 512], [5, 6, 400, 450], [0, 0, 0, 0])):
        q, k, v = _inputs(("graph", i), T, H, Hkv, dh)
        dq.copy_(ref.to_dev(q)), dk.copy_(ref.to_dev(k)), dv.copy_(ref.to_dev(v)), off.copy_(_i32(*at))
        o.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        _check(ref.from_dev(o), q, k, v, at)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        o2 = torch.full_like(o, 5.0)
        _vb().vla_op_attention_packed(dq, dk, dv, _i32(3, 200, 500), o2)
    s.synchronize()
    _check(ref.from_dev(o2), q, k, v, [3, 200, 500])
