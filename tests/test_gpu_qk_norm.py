"""Per-head norm and rotary embedding against float64."""
import numpy as np
import pytest

import w4kv4_ref as ref

pytestmark = pytest.mark.gpu


def _tables(n, dh):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, dh, 2) / dh)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _check(got, want, mag):
    """One bf16 rounding (2^-9 relative, asserted at 2^-8 with the fp32 part
    inside it) of a difference of two products, each with the norm's fp32
    error (a dozen roundings) in front of it."""
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * mag + 1e-38).all()


@pytest.mark.parametrize("B,L,H,Hkv,dh", [(1, 1, 1, 1, 64), (2, 3, 14, 2, 64), (1, 37, 32, 32, 128), (3, 5, 5, 1, 128),
                                          (1, 130, 7, 7, 64), (4, 1, 40, 8, 128), (1, 700, 2, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_qk_norm_rope(B, L, H, Hkv, dh, dtype):
    import torch
    from paper_2608_14586_amd import binding as vb
    rows = ref.normal(("qk", B, L, H, dh), (B, L, H + 2 * Hkv, dh), 2.0)
    rng = np.random.default_rng(L)
    gq, gk = (rng.uniform(0.5, 1.5, dh).astype(np.float32) for _ in range(2))
    cos, sin = _tables(2 * L + 50, dh)
    pos = rng.integers(0, len(cos), (B, L)).astype(np.int32)
    dev = ref.to_dev(rows, dtype)  # q and k in place inside the fused projection's rows
    q_out = torch.empty((B, H, L, dh), dtype=torch.bfloat16, device="cuda")  # heads before tokens
    k_out = torch.empty((B, L, Hkv, dh), dtype=torch.bfloat16, device="cuda")
    t = [torch.from_numpy(a).cuda() for a in (gq, gk, cos, sin, pos)]
    vb.vla_op_qk_norm_rope(dev[:, :, :H], dev[:, :, H:H + Hkv], t[0], t[1], 1e-6, t[2], t[3], t[4],
                           q_out.transpose(1, 2), k_out)
    c, s = cos[pos].astype(np.float64), sin[pos].astype(np.float64)
    for got, x, g in ((ref.from_dev(q_out.transpose(1, 2)), rows[:, :, :H], gq), (ref.from_dev(k_out), rows[:, :, H:H + Hkv], gk)):
        n = ref.head_norm_rope(x, g.astype(np.float64), 1e-6, None, None)
        mag = np.abs(n) + np.abs(np.concatenate(np.split(n, 2, -1)[::-1], -1))
        _check(got, ref.head_norm_rope(x, g.astype(np.float64), 1e-6, c, s), mag)


def test_parts_in_place_and_padding():
    """Norm alone, rotation alone, neither (a copy), in place, and tokens whose
    position is no row of the tables: they stay as they were."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, L, H, dh = 2, 4, 3, 64
    x = ref.normal(("parts",), (B, L, 2 * H, dh))
    cos, sin = _tables(9, dh)
    tc, ts = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    g = np.linspace(0.5, 1.5, dh).astype(np.float32)
    tg = torch.from_numpy(g).cuda()
    q, k = x[:, :, :H], x[:, :, H:]

    def call(gq, gk, rot, pos=None):
        d = ref.to_dev(x)
        p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
        vb.vla_op_qk_norm_rope(d[:, :, :H], d[:, :, H:], gq, gk, 1e-6, tc if rot else None, ts if rot else None, p,
                               d[:, :, :H], d[:, :, H:])
        y = ref.from_dev(d)
        return y[:, :, :H], y[:, :, H:]

    c, s = cos[:L].astype(np.float64)[None], sin[:L].astype(np.float64)[None]
    yq, yk = call(None, None, False)
    assert np.array_equal(yq, q) and np.array_equal(yk, k)
    yq, yk = call(tg, None, True)  # positions 0 .. L - 1
    _check(yq, ref.head_norm_rope(q, g.astype(np.float64), 1e-6, c, s), 8.0)
    _check(yk, ref.head_norm_rope(k, None, 0, c, s), 8.0)
    yq, yk = call(None, tg, False)
    assert np.array_equal(yq, q)
    _check(yk, ref.head_norm_rope(k, g.astype(np.float64), 1e-6, None, None), 8.0)
    pos = [[3, -1, 8, 9], [2 ** 31 - 1, 0, -2 ** 31, 5]]
    yq, yk = call(tg, tg, True, pos)
    for b in range(B):
        for t in range(L):
            p = pos[b][t]
            if not 0 <= p < 9:
                assert np.array_equal(yq[b, t], q[b, t]) and np.array_equal(yk[b, t], k[b, t])
            else:
                _check(yq[b, t], ref.head_norm_rope(q[b, t], g.astype(np.float64), 1e-6, cos[p].astype(np.float64),
                                                    sin[p].astype(np.float64)), 8.0)


def test_extremes():
    """A row of zeros stays zero, tiny and large rows are normalised, and a row
    that is not finite reaches no other."""
    import torch
    from paper_2608_14586_amd import binding as vb
    H, dh = 6, 128
    x = ref.normal(("ext",), (1, 1, H, dh))
    x[0, 0, 0] = 0
    x[0, 0, 1] = ref.bf16(x[0, 0, 1] * 1e-6)
    x[0, 0, 2] = ref.bf16(x[0, 0, 2] * 1e18)
    x[0, 0, 3, 5] = np.nan
    x[0, 0, 4, 100] = np.inf
    out = torch.zeros((1, 1, H, dh), dtype=torch.bfloat16, device="cuda")
    k = ref.to_dev(x[:, :, :1])
    g = torch.ones(dh, device="cuda")
    vb.vla_op_qk_norm_rope(ref.to_dev(x), k, g, g, 1e-12, None, None, None, out, torch.empty_like(k))
    got = ref.from_dev(out)[0, 0]
    want = ref.head_norm_rope(x[0, 0], np.ones(dh), 1e-12, None, None)
    assert (got[0] == 0).all()
    for h in (1, 2, 5):
        _check(got[h], want[h], 8.0)
    assert np.isnan(got[3]).all() and np.isnan(got[4, 100])
