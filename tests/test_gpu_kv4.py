"""The 4-bit KV cache and the attention over it, against float64."""
import numpy as np
import pytest

import synth
import w4kv4_ref as ref

pytestmark = pytest.mark.gpu


def _cache(B, Hkv, L_cap, dh, byte=0):
    import torch
    from paper_2608_14586_amd import binding as vb
    return torch.full((vb.vla_op_kv4_bytes(B, Hkv, L_cap, dh),), byte, dtype=torch.uint8, device="cuda")


def _i32(*v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _kv(tag, B, L, Hkv, dh):
    k, v = (ref.normal((n,) + tag, (B, L, Hkv, dh)) for n in "kv")
    return ref.bf16(k * (1 + 4 * (np.arange(dh) % 23 == 0))), v  # a few strong channels


def _load(cache, L_cap, B, L, Hkv, dh, start=None, count=None, fill=0.0):
    import torch
    from paper_2608_14586_amd import binding as vb
    k = torch.full((B, L, Hkv, dh), fill, dtype=torch.bfloat16, device="cuda")
    v = torch.full((B, L, Hkv, dh), fill, dtype=torch.bfloat16, device="cuda")
    vb.vla_op_kv4_load(cache, L_cap, start, count, k, v)
    return ref.from_dev(k), ref.from_dev(v)


@pytest.mark.parametrize("B,L,Hkv,dh,start", [(1, 1, 1, 64, 0), (1, 1, 1, 128, 31), (2, 33, 2, 64, 5), (1, 64, 3, 128, 0),
                                              (3, 40, 1, 128, 63), (2, 200, 4, 64, 17), (1, 31, 8, 128, 32)])
def test_store_and_load(B, L, Hkv, dh, start):
    """Every row comes back as the value its 4 bits stand for, to the last bit
    (the quantisation's ties included: bf16 values over a range of 15 steps hit
    many), and every other row of a cache full of something stays."""
    import torch
    from paper_2608_14586_amd import binding as vb
    L_cap = (start + L + 32 + 31) // 32 * 32
    k, v = _kv((B, L, Hkv, dh), B, L, Hkv, dh)
    v = np.round(v * 4) / 4  # coarse values: quotients on the borders between codes
    cache = _cache(B, Hkv, L_cap, dh)
    cache.copy_(torch.from_numpy(np.random.default_rng(B).integers(0, 63, cache.numel(), dtype=np.uint8)))
    before = _load(cache, L_cap, B, L_cap, Hkv, dh)
    st = _i32(*[start + (b % 2) for b in range(B)])
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), st, None, cache, L_cap)
    after = _load(cache, L_cap, B, L_cap, Hkv, dh)
    for x, old, new in ((k, before[0], after[0]), (v, before[1], after[1])):
        want = old.copy()
        for b in range(B):
            at = start + b % 2
            want[b, at:at + L] = ref.bf16(ref.cached(x[b]))
        assert np.array_equal(new, want)
    got = _load(cache, L_cap, B, L, Hkv, dh, st)
    assert np.array_equal(got[0], ref.bf16(ref.cached(k))) and np.array_equal(got[1], ref.bf16(ref.cached(v)))


def test_store_in_pieces_equals_whole():
    """Tokens stored one by one, in odd pieces and at once give the same bytes."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, L, Hkv, dh, L_cap = 2, 77, 2, 128, 96
    k, v = _kv(("pieces",), B, L, Hkv, dh)
    dk, dv = ref.to_dev(k), ref.to_dev(v)
    whole = _cache(B, Hkv, L_cap, dh)
    vb.vla_op_kv4_store(dk, dv, None, None, whole, L_cap)
    for sizes in ([1] * L, [5, 1, 31, 33, 7], [32, 45]):
        c, at = _cache(B, Hkv, L_cap, dh), 0
        for n in sizes:
            vb.vla_op_kv4_store(dk[:, at:at + n], dv[:, at:at + n], _i32(at, at), None, c, L_cap)
            at += n
        assert at == L and torch.equal(c, whole), sizes


def test_store_bounds_counts_and_strides():
    """Positions outside the cache and tokens past a sequence's count are left
    out, in both directions; heads before tokens, rows of a fused projection."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, L, Hkv, dh, L_cap = 7, 50, 2, 64, 64
    k, v = _kv(("bounds",), B, L, Hkv, dh)
    start = [-20, 40, 64, -60, 10, 2 ** 31 - 1, -2 ** 31]
    count = [L, L, L, L, 0, L, 999]
    cache = _cache(B, Hkv, L_cap, dh, 17)
    before = _load(cache, L_cap, B, L_cap, Hkv, dh)
    rows = torch.zeros((B, L, 5 * Hkv, dh), dtype=torch.bfloat16, device="cuda")
    rows[:, :, 2 * Hkv:3 * Hkv] = ref.to_dev(k)
    vh = ref.to_dev(v).transpose(1, 2).contiguous()  # [B][Hkv][L][dh]
    vb.vla_op_kv4_store(rows[:, :, 2 * Hkv:3 * Hkv], vh.transpose(1, 2), _i32(*start), _i32(*count), cache, L_cap)
    after = _load(cache, L_cap, B, L_cap, Hkv, dh)
    for x, old, new in ((k, before[0], after[0]), (v, before[1], after[1])):
        want = old.copy()
        for b in range(B):
            for t in range(min(max(count[b], 0), L)):
                if 0 <= start[b] + t < L_cap:
                    want[b, start[b] + t] = ref.bf16(ref.cached(x[b, t]))
        assert np.array_equal(new, want)
    got = _load(cache, L_cap, B, L, Hkv, dh, _i32(*start), _i32(*count), fill=3.0)
    for x, new in ((k, got[0]), (v, got[1])):
        for b in range(B):
            for t in range(L):
                there = t < min(max(count[b], 0), L) and 0 <= start[b] + t < L_cap
                assert np.array_equal(new[b, t], ref.bf16(ref.cached(x[b, t])) if there else np.full((Hkv, dh), 3.0))


def test_quantiser_extremes():
    """Constant groups, the largest and smallest numbers, infinities and NaN
    (their group reads back as NaN, no other one does)."""
    from paper_2608_14586_amd import binding as vb
    dh = 128
    big = 3.3895313892515355e38  # the largest bf16
    x = ref.normal(("extremes",), (1, 9, 1, dh))
    x[0, 0, 0, :32] = 2.5
    x[0, 0, 0, 32:64] = 0.0
    x[0, 1, 0, :32] = np.where(np.arange(32) % 2, big, -big)
    x[0, 2, 0, :32] = ref.bf16(x[0, 2, 0, :32] * 2.0 ** -110)  # below the least range
    x[0, 3, 0, :32] = ref.bf16(x[0, 3, 0, :32] * 2.0 ** -95)
    x[0, 4, 0, 40] = np.nan
    x[0, 5, 0, 70] = np.inf
    x[0, 6, 0, 0] = -np.inf
    x[0, 7, 0, :32] = np.arange(32) - 16.0  # quotients on and off the borders
    x[0, 8, 0, :32] = np.where(np.arange(32) == 3, 100.0, 100.0 + 0.5)  # far from zero
    cache = _cache(1, 1, 32, dh)
    vb.vla_op_kv4_store(ref.to_dev(x), ref.to_dev(-x), None, None, cache, 32)
    got = _load(cache, 32, 1, 9, 1, dh)
    for y, sign in ((got[0], 1), (got[1], -1)):
        want = ref.bf16(ref.cached(sign * x))
        assert np.array_equal(np.isnan(y), np.isnan(want))
        assert np.array_equal(y[~np.isnan(y)], want[~np.isnan(want)])
    assert np.isnan(got[0]).sum() == 3 * 32


# ------------------------------------------------------------------ attention

def _attend(q, cache, L_cap, Hkv, lens, max_len, window=0, sinks=0, stream=None):
    import torch
    from paper_2608_14586_amd import binding as vb
    B, Lq, H, dh = q.shape
    n = vb.vla_op_attention_kv4_scratch(B, Lq, H, Hkv, dh, max_len, window, sinks)
    scratch = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None  # NaN everywhere
    o = torch.full((B, Lq, H, dh), 11.0, dtype=torch.bfloat16, device="cuda")
    vb.vla_op_attention_kv4(q, cache, L_cap, Hkv, _i32(*lens), o, max_len, window, sinks, scratch, stream)
    return ref.from_dev(o)


def _check(got, q, k, v, lens, window, sinks):
    """Against float64 over the cached values.  One bf16 rounding of the result
    (2^-8 of it, a factor 2); a score's fp32 error moves its weight: its sums
    run over (16 + c) s q and m q, a hundred times a score's size in the cases
    here, a few dozen roundings of 2^-24 each: below 2^-11 of sum p |v| with a
    margin; the weights' 16-bit significand (2^-17) multiplies at most 31 steps
    of a value, below 2^-11 of the largest value."""
    kc, vc = ref.cached(k), ref.cached(v)
    for b in range(len(lens)):
        want, mag = ref.attention(q[b], kc[b], vc[b], lens[b], window, sinks)
        top = np.abs(vc[b, :lens[b]]).max() if lens[b] else 0.0
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * (mag + top)
        err = np.abs(got[b] - want)
        assert (err <= bound).all(), (b, np.unravel_index(np.argmax(err - bound), err.shape), (err - bound).max())


CASES = [
    # B, Lq, H, Hkv, dh, lens, window, sinks
    (1, 1, 1, 1, 64, [1], 0, 0), (1, 1, 4, 4, 128, [31], 0, 0), (2, 1, 8, 2, 64, [32, 33], 0, 0),
    (3, 1, 14, 2, 64, [0, 1, 700], 0, 0), (2, 1, 32, 8, 128, [257, 1000], 0, 0), (1, 1, 16, 1, 128, [2049], 0, 0),
    (1, 1, 40, 2, 64, [300], 0, 0),  # 20 queries a KV head: two tiles
    (2, 3, 8, 2, 128, [2, 100], 0, 0),  # a query before the first token: nothing to see
    (1, 5, 14, 2, 64, [64], 0, 0), (2, 16, 4, 4, 64, [16, 333], 0, 0), (1, 37, 6, 2, 128, [90], 0, 0),
    (2, 1, 8, 2, 64, [50, 500], 100, 0), (2, 1, 8, 8, 128, [500, 3], 33, 4), (1, 1, 4, 1, 128, [1500], 1, 0),
    (1, 1, 4, 1, 128, [1500], 1, 1), (2, 4, 28, 4, 128, [1111, 40], 64, 70), (1, 9, 4, 2, 64, [777], 200, 5),
    (1, 3, 4, 2, 64, [20], 5, 100), (1, 1, 2, 1, 64, [6000], 0, 0), (9, 1, 2, 1, 128, list(range(1, 200, 24)), 0, 0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case):
    from paper_2608_14586_amd import binding as vb
    B, Lq, H, Hkv, dh, lens, window, sinks = CASES[case]
    n = max(lens)
    k, v = _kv((case,), B, max(n, 1), Hkv, dh)
    q = ref.normal(("q", case), (B, Lq, H, dh))
    for L_cap, max_len in (((n + 31) // 32 * 32 or 32, n), ((n + 95) // 32 * 32 + 2048, n + 64)):
        cache = _cache(B, Hkv, L_cap, dh, 255)  # unwritten rows: NaN
        vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, _i32(*lens), cache, L_cap)
        got = _attend(ref.to_dev(q), cache, L_cap, Hkv, lens, max_len, window, sinks)
        _check(got, q, k, v, lens, window, sinks)


def test_attention_keeps_hidden_rows_out():
    """Keys and values that a query may not see (later tokens, tokens before
    its window) can hold NaN; the query's result does not change by a bit."""
    from paper_2608_14586_amd import binding as vb
    B, Lq, H, Hkv, dh, n, window, sinks = 1, 4, 8, 2, 128, 300, 70, 3
    k, v = _kv(("hidden",), B, n, Hkv, dh)
    q = ref.to_dev(ref.normal(("hq",), (B, Lq, H, dh)))
    clean, dirty = _cache(B, Hkv, 320, dh), _cache(B, Hkv, 320, dh, 255)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, clean, 320)
    k[0, -1], v[0, -1] = np.nan, np.nan  # only the last query sees it
    k[0, 3:n - Lq - window + 1], v[0, 3:n - Lq - window + 1] = np.nan, np.nan  # between sinks and the first query's window
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, dirty, 320)
    a = _attend(q, clean, 320, Hkv, [n], n, window, sinks)
    b = _attend(q, dirty, 320, Hkv, [n], n, window, sinks)
    assert np.array_equal(a[0, :3], b[0, :3])
    assert np.isnan(b[0, 3]).all()


@pytest.mark.parametrize("byte", [0x7e, 0x01, 0x80, 0xc3])
def test_attention_beside_unwritten_rows(byte):
    """The block that holds a sequence's last tokens also holds rows that were
    never written; whatever numbers they look like (steps of 8e37 or 2e-38,
    negative ones), the result is that of a clean cache, to the last bit."""
    from paper_2608_14586_amd import binding as vb
    B, Lq, H, Hkv, dh = 2, 2, 8, 2, 64
    lens = [37, 3]
    k, v = _kv(("beside",), B, 37, Hkv, dh)
    q = ref.to_dev(ref.normal(("bsq",), (B, Lq, H, dh)))
    out = []
    for fill in (0, byte):
        cache = _cache(B, Hkv, 64, dh, fill)
        vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, _i32(*lens), cache, 64)
        out.append(_attend(q, cache, 64, Hkv, lens, 37))
    assert np.array_equal(out[0], out[1])
    _check(out[1], ref.from_dev(q), k, v, lens, 0, 0)


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -20, 2.0 ** 30, 2.0 ** 100])
def test_attention_at_any_size_of_values(scale):
    """Values far from one, and groups whose steps differ by 2^60 or are zero
    in their first tokens: every group's result is as exact as its own values'
    size allows."""
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh, n = 1, 4, 2, 128, 200
    k, v = _kv(("sizes",), B, n, Hkv, dh)
    v *= scale
    v[..., 32:64] *= 2.0 ** -40
    v[:, :70, :, 64:96] = scale  # constant at first
    v[:, :, :, 96:] = np.where(np.arange(n)[:, None, None] < 100, 2.0 ** -30, 1.0) * v[:, :, :, 96:]
    q = ref.normal(("szq",), (B, 1, H, dh))
    cache = _cache(B, Hkv, 224, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 224)
    got = _attend(ref.to_dev(q), cache, 224, Hkv, [n], n)
    for g in range(4):  # each group against its own size
        at = slice(32 * g, 32 * g + 32)
        kc, vc = ref.cached(k), ref.cached(v)
        want, mag = ref.attention(q[0], kc[0], vc[0], n, 0, 0)
        top = np.abs(vc[0, ..., at]).max()
        assert (np.abs(got[0] - want)[..., at] <= 2.0 ** -8 * np.abs(want[..., at]) + 2.0 ** -11 * (mag[..., at] + top)).all(), g


def test_attention_lens_are_cut():
    """Lengths below 0 count as 0 and above max_len as max_len."""
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh = 4, 4, 2, 64
    k, v = _kv(("cut",), B, 96, Hkv, dh)
    q = ref.normal(("cutq",), (B, 1, H, dh))
    cache = _cache(B, Hkv, 96, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 96)
    got = _attend(ref.to_dev(q), cache, 96, Hkv, [-5, 70, 1000, 2 ** 31 - 1], 80)
    _check(got, q, k, v, [0, 70, 80, 80], 0, 0)


def test_attention_strides_streams_and_graph():
    """q inside a fused row, o with heads before tokens, a side stream, and a
    captured call replayed as the cache grows: each equals the plain call."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, Lq, H, Hkv, dh, n = 2, 2, 8, 2, 128, 1500
    k, v = _kv(("strides",), B, n, Hkv, dh)
    q = ref.normal(("sq",), (B, Lq, H, dh))
    cache = _cache(B, Hkv, 1504, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 1504)
    lens = [1500, 901]
    plain = _attend(ref.to_dev(q), cache, 1504, Hkv, lens, n)
    rows = torch.zeros((B, Lq, H + 2 * Hkv, dh), dtype=torch.bfloat16, device="cuda")
    rows[:, :, :H] = ref.to_dev(q)
    o = torch.zeros((B, H, Lq, dh), dtype=torch.bfloat16, device="cuda")
    nbytes = vb.vla_op_attention_kv4_scratch(B, Lq, H, Hkv, dh, n)
    assert nbytes > 0
    scratch = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    dl = _i32(*lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    args = (rows[:, :, :H], cache, 1504, Hkv, dl, o.transpose(1, 2), n, 0, 0, scratch)
    vb.vla_op_attention_kv4(*args, stream=side.cuda_stream)
    side.synchronize()
    assert np.array_equal(ref.from_dev(o.transpose(1, 2)), plain)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        vb.vla_op_attention_kv4(*args, stream=torch.cuda.current_stream().cuda_stream)
    for lens in ([1500, 901], [3, 0], [700, 1499], [1, 2]):
        dl.copy_(_i32(*lens))
        o.fill_(4.0)
        scratch.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        got = ref.from_dev(o.transpose(1, 2))
        assert np.array_equal(got, _attend(ref.to_dev(q), cache, 1504, Hkv, lens, n)), lens
        _check(got, q, k, v, lens, 0, 0)


def test_offsets_past_32_bits():
    """Two heads of 2^24 tokens (5.4 GB): rows at the far end of the second
    come back, and a window there is attended to."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh, cap, n = 1, 4, 2, 128, 1 << 24, 70
    k, v = _kv(("far",), B, n, Hkv, dh)
    q = ref.normal(("farq",), (B, 1, H, dh))
    cache = torch.empty(vb.vla_op_kv4_bytes(B, Hkv, cap, dh), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), _i32(cap - n), None, cache, cap)
    got = _load(cache, cap, B, n, Hkv, dh, _i32(cap - n))
    assert np.array_equal(got[0], ref.bf16(ref.cached(k))) and np.array_equal(got[1], ref.bf16(ref.cached(v)))
    out = _attend(ref.to_dev(q), cache, cap, Hkv, [cap], cap, 60, 0)
    # the last 60 of these tokens, as a sequence of their own
    _check(out, q, k, v, [n], 60, 0)


def test_batch_does_not_change_a_sequence():
    """A sequence's cache and result are the same bytes next to other sequences,
    where both calls split the keys alike."""
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh, n = 3, 8, 2, 64, 100
    k, v = _kv(("batch",), B, n, Hkv, dh)
    q = ref.to_dev(ref.normal(("bq",), (B, 1, H, dh)))
    cache = _cache(B, Hkv, 128, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 128)
    whole = _attend(q, cache, 128, Hkv, [n] * B, n)
    each = cache.numel() // B
    for b in range(B):
        assert np.array_equal(_attend(q[b:b + 1], cache[b * each:(b + 1) * each], 128, Hkv, [n], n)[0], whole[b])


def test_tensors_that_do_not_fit():
    """Wrong types, shapes, sizes, devices and strides raise before any launch,
    and a scratch that is too small is VLA_ERR_SHAPE."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, L, H, Hkv, dh, cap = 2, 40, 4, 2, 64, 2048
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, q, cache, lens = bf(B, L, Hkv, dh), bf(B, 1, H, dh), _cache(B, Hkv, cap, dh), _i32(40, 40)
    scratch = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    tab = torch.zeros((4, dh // 2), device="cuda")
    store = lambda **c: vb.vla_op_kv4_store(**{**dict(k=k, v=k, start=None, count=lens, cache=cache, L_cap=cap), **c})  # noqa: E731
    attend = lambda **c: vb.vla_op_attention_kv4(**{**dict(q=q, cache=cache, L_cap=cap, Hkv=Hkv, lens=lens, o=q.clone(), max_len=cap, scratch=scratch), **c})  # noqa: E731
    rope = lambda **c: vb.vla_op_qk_norm_rope(**{**dict(q=q, k=bf(B, 1, Hkv, dh), gq=None, gk=None, eps=0.0, cos=tab, sin=tab, pos=None, q_out=q, k_out=bf(B, 1, Hkv, dh)), **c})  # noqa: E731
    store(), attend(), rope()
    for bad in (lambda: store(v=k.float()), lambda: store(v=k[:, :39]), lambda: store(k=k.transpose(2, 3)), lambda: store(count=lens.long()),
                lambda: store(count=lens[:1]), lambda: store(cache=cache[:-1]), lambda: store(cache=cache.cpu()), lambda: store(L_cap=cap + 32),
                lambda: store(k=k[0]), lambda: store(start=_i32(0, 0, 0, 0)[::2]), lambda: attend(lens=None), lambda: attend(lens=lens.float()),
                lambda: attend(o=q.float()), lambda: attend(o=bf(B, 1, H, dh + 64)[..., ::2][..., :dh]), lambda: attend(q=q.cpu()),
                lambda: attend(Hkv=4), lambda: attend(max_len=1 << 40), lambda: rope(sin=tab[:2]), lambda: rope(gq=tab[0]),
                lambda: rope(pos=torch.zeros((B, 1), dtype=torch.int64, device="cuda")), lambda: rope(k=k), lambda: rope(q=q.half()),
                lambda: store(stream="s"), lambda: attend(stream=-1.5)):
        with pytest.raises(ValueError):
            bad()
    need = vb.vla_op_attention_kv4_scratch(B, 1, H, Hkv, dh, cap)
    assert need > 0
    for small in (None, scratch[:need - 4]):
        with pytest.raises(vb.VlaError) as e:
            attend(scratch=small)
        assert e.value.name == "VLA_ERR_SHAPE"
    with pytest.raises(vb.VlaError) as e:
        attend(max_len=cap + 1)
    assert e.value.name == "VLA_ERR_SHAPE"
    torch.cuda.synchronize()


# ------------------------------------------------------------------- together

@pytest.mark.parametrize("H,Hkv,dh,window", [(14, 2, 64, 0), (4, 4, 128, 40)])
def test_decoder_block_in_4_bits(H, Hkv, dh, window):
    """A decoder block of new tokens with 4-bit weights over a 4-bit cache, step
    by step: norm, QKV, head norms with rotary embedding, cache, attention,
    output projection into the residual, norm, gate/up with SwiGLU, down --
    against the same steps in float64, rounded to bf16 where the operators
    round.  A rounding that falls to the other side moves a later step's input
    by one bf16 step (2^-8) and a cached code by one level, so the residual's
    update is compared as a whole: 2e-2 of its norm, twice what all roundings
    to bf16 and one flipped level in a hundred can give."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, d, F, steps, past, group = 2, 256, 352, 4, 75, 64
    rng = np.random.default_rng(synth.seed_of("block", H, dh))

    def weight(N, K):
        codes = rng.integers(0, 16, (N, K), dtype=np.uint8)
        s = ref.bf16(rng.uniform(0.5, 1.5, (N, -(-K // group))) / (4.6 * np.sqrt(K)))
        Wp = torch.empty(vb.vla_op_w4_packed_bytes(N, K, group), dtype=torch.uint8, device="cuda")
        vb.vla_op_w4_pack(torch.from_numpy(codes).cuda(), ref.to_dev(s), None, Wp, group)
        return Wp, ref.w4_weights(codes, s, None, group).T

    nh = H + 2 * Hkv
    wqkv, wo, wup, wdown = weight(nh * dh, d), weight(d, H * dh), weight(2 * F, d), weight(d, F)
    g1, g2, gq, gk = (rng.uniform(0.5, 1.5, n).astype(np.float32) for n in (d, d, dh, dh))
    t1, t2, tq, tk = (torch.from_numpy(g).cuda() for g in (g1, g2, gq, gk))
    ang = np.arange(128)[:, None] * 10000.0 ** (-np.arange(0, dh, 2) / dh)
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    tc, ts = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    k0, v0 = _kv(("block", H), B, past, Hkv, dh)
    cap, max_len = 128, past + steps
    cache = _cache(B, Hkv, cap, dh)
    vb.vla_op_kv4_store(ref.to_dev(k0), ref.to_dev(v0), None, None, cache, cap)
    kc, vc = [k0], [v0]
    rms = lambda x, g: ref.bf16(x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * g)  # noqa: E731
    bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    xn, rows, q, k, o, a = bf(B, d), bf(B, nh * dh), bf(B, 1, H, dh), bf(B, 1, Hkv, dh), bf(B, 1, H, dh), bf(B, F)
    n = vb.vla_op_attention_kv4_scratch(B, 1, H, Hkv, dh, max_len, window, 2)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        at = past + step
        h0 = synth.normal_f32(synth.seed_of("blockh", step, H), (B, d))
        h = torch.from_numpy(h0.copy()).cuda()
        pos, start, lens = _i32(*[at] * B).view(B, 1), _i32(*[at] * B), _i32(*[at + 1] * B)
        vb.vla_op_norm_bf16(h, t1, None, 1e-6, xn, B, d)
        vb.vla_op_gemv_w4(xn, wqkv[0], None, rows, nh * dh, group)
        heads = rows.view(B, 1, nh, dh)
        vb.vla_op_qk_norm_rope(heads[:, :, :H], heads[:, :, H:H + Hkv], tq, tk, 1e-6, tc, ts, pos, q, k)
        vb.vla_op_kv4_store(k, heads[:, :, H + Hkv:], start, None, cache, cap)
        vb.vla_op_attention_kv4(q, cache, cap, Hkv, lens, o, max_len, window, 2, scratch)
        vb.vla_op_gemv_w4(o.view(B, H * dh), wo[0], h, h, d, group)
        vb.vla_op_norm_bf16(h, t2, None, 1e-6, xn, B, d)
        vb.vla_op_gemv_w4(xn, wup[0], None, a, 2 * F, group, True)
        vb.vla_op_gemv_w4(a, wdown[0], h, h, d, group)

        y = ref.bf16(rms(h0.astype(np.float64), g1) @ wqkv[1]).reshape(B, 1, nh, dh)
        c, s = cos[None, at:at + 1].astype(np.float64), sin[None, at:at + 1].astype(np.float64)
        rq = ref.bf16(ref.head_norm_rope(y[:, :, :H], gq.astype(np.float64), 1e-6, c, s))
        kc.append(ref.bf16(ref.head_norm_rope(y[:, :, H:H + Hkv], gk.astype(np.float64), 1e-6, c, s)))
        vc.append(y[:, :, H + Hkv:])
        kk, vv = ref.cached(np.concatenate(kc, 1)), ref.cached(np.concatenate(vc, 1))
        ro = np.stack([ref.attention(rq[b], kk[b], vv[b], at + 1, window, 2)[0] for b in range(B)])
        want = h0 + ref.bf16(ro).reshape(B, H * dh) @ wo[1]
        up = rms(want, g2) @ wup[1]
        want = want + ref.bf16(up[:, :F] / (1 + np.exp(-up[:, :F])) * up[:, F:]) @ wdown[1]
        got = ref.from_dev(h)
        assert np.linalg.norm(got - want) <= 2e-2 * np.linalg.norm(want - h0), step


def test_decode_step_in_a_graph():
    """Head norms, cache append, attention and the output projection of a decode
    step captured once, its position on the device: every replay is the eager
    step, to the last bit, as the cache grows over a block's end."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh, d, cap, group, past = 2, 8, 2, 128, 256, 96, 64, 29
    rng = np.random.default_rng(9)
    codes = torch.from_numpy(rng.integers(0, 16, (d, H * dh), dtype=np.uint8)).cuda()
    s = ref.to_dev(rng.uniform(0.002, 0.01, (d, H * dh // group)))
    Wp = torch.empty(vb.vla_op_w4_packed_bytes(d, H * dh, group), dtype=torch.uint8, device="cuda")
    vb.vla_op_w4_pack(codes, s, None, Wp, group)
    ang = np.arange(cap)[:, None] * 10000.0 ** (-np.arange(0, dh, 2) / dh)
    tc, ts = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    g = torch.from_numpy(rng.uniform(0.5, 1.5, dh).astype(np.float32)).cuda()
    k0, v0 = _kv(("graph",), B, past, Hkv, dh)
    bf = lambda *sh: torch.zeros(sh, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    rows, q, k, o = bf(B, 1, H + 2 * Hkv, dh), bf(B, 1, H, dh), bf(B, 1, Hkv, dh), bf(B, 1, H, dh)
    h = torch.zeros((B, d), device="cuda")
    pos, lens = _i32(past, past), _i32(past + 1, past + 1)
    caches = [_cache(B, Hkv, cap, dh) for _ in range(2)]
    n = vb.vla_op_attention_kv4_scratch(B, 1, H, Hkv, dh, cap)
    scratch = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
    for c in caches:
        vb.vla_op_kv4_store(ref.to_dev(k0), ref.to_dev(v0), None, None, c, cap)

    def step(cache, stream):
        vb.vla_op_qk_norm_rope(rows[:, :, :H], rows[:, :, H:H + Hkv], g, g, 1e-6, tc, ts, pos.view(B, 1), q, k, stream)
        vb.vla_op_kv4_store(k, rows[:, :, H + Hkv:], pos, None, cache, cap, stream)
        vb.vla_op_attention_kv4(q, cache, cap, Hkv, lens, o, cap, 0, 0, scratch, stream)
        vb.vla_op_gemv_w4(o.view(B, H * dh), Wp, h, h, d, group, False, stream)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], torch.cuda.current_stream().cuda_stream)
    for t in range(6):
        rows.copy_(ref.to_dev(ref.normal(("graphrows", t), rows.shape)))
        pos.fill_(past + t)
        lens.fill_(past + t + 1)
        h.fill_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        got = h.clone()
        h.fill_(0.25)
        step(caches[1], None)
        torch.cuda.synchronize()
        assert torch.equal(got, h) and torch.equal(caches[0], caches[1]), t


def test_two_streams_at_once():
    """Two attentions that run at the same time, each with its own scratch."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, H, Hkv, dh, n = 1, 32, 8, 128, 3000
    k, v = _kv(("two",), B, n, Hkv, dh)
    cache = _cache(B, Hkv, 3008, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 3008)
    qs = [ref.to_dev(ref.normal(("twoq", i), (B, 1, H, dh))) for i in range(2)]
    lens = _i32(n)
    need = vb.vla_op_attention_kv4_scratch(B, 1, H, Hkv, dh, n)
    assert need > 0
    alone = [_attend(q, cache, 3008, Hkv, [n], n) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    scratch = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in qs]
    outs = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, s, st in zip(qs, outs, scratch, streams):
            vb.vla_op_attention_kv4(q, cache, 3008, Hkv, lens, o, n, 0, 0, s, st.cuda_stream)
    torch.cuda.synchronize()
    for o, a in zip(outs, alone):
        assert np.array_equal(ref.from_dev(o), a)


def test_a_query_that_is_not_finite():
    """reaches no other query of its tile, whatever the split."""
    B, Lq, H, Hkv, dh, n = 1, 3, 8, 2, 128, 700
    k, v = _kv(("nan",), B, n, Hkv, dh)
    from paper_2608_14586_amd import binding as vb
    cache = _cache(B, Hkv, 704, dh)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, None, cache, 704)
    q = ref.normal(("nanq",), (B, Lq, H, dh))
    want = _attend(ref.to_dev(q), cache, 704, Hkv, [n], n)
    for bad in (np.nan, np.inf):
        x = q.copy()
        x[0, 1, 2, 5] = bad
        got = _attend(ref.to_dev(x), cache, 704, Hkv, [n], n)
        assert np.isnan(got[0, 1, 2]).all()
        got[0, 1, 2] = want[0, 1, 2]
        assert np.isfinite(want).all() and np.abs(got - want).max() <= 2.0 ** -7 * np.abs(want).max()


def test_steps_that_fall_between_two_bf16_numbers():
    """Ranges of 15 times an odd number of half bf16 steps: (max - min) / 15 is a
    tie, and the step is what the product in fp32 rounds to."""
    odd = np.arange(257, 512, 2)  # 9 bits, the last one set
    k = np.zeros((1, 128, 1, 64))
    k[0, :, 0, 0], k[0, :, 0, 32] = odd * 15 / 64.0, -odd * 15 / 64.0  # 13 bits: reached by two bf16 numbers each
    hi = ref.bf16(k[..., 0:1])
    k[..., 1:2], k[..., 0:1] = hi - k[..., 0:1], hi
    k[..., 33:34], k[..., 32:33] = -hi - k[..., 32:33], -hi
    k[..., 5:30] = hi * np.linspace(0, 1, 25)
    k[..., 37:62] = -hi * np.linspace(0, 1, 25)
    k = ref.bf16(k)
    from paper_2608_14586_amd import binding as vb
    cache = _cache(1, 1, 128, 64)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(k), None, None, cache, 128)
    a, b = ref.to_dev(k * 0), ref.to_dev(k * 0)
    vb.vla_op_kv4_load(cache, 128, None, None, a, b)
    want = ref.bf16(ref.cached(k))
    assert np.array_equal(ref.from_dev(a), want) and np.array_equal(ref.from_dev(b), want)


@pytest.mark.parametrize("B,Lq,max_len,lens", [(2, 1, 0, 0), (2, 1, 0, 9), (1, 5, 3, 3), (300, 1, 40, 37), (3, 70, 64, 64)])
def test_attention_at_the_ends_of_its_sizes(B, Lq, max_len, lens):
    """No tokens at all, a cut to none, more queries than tokens, many sequences."""
    from paper_2608_14586_amd import binding as vb
    H, Hkv, dh = 4, 2, 64
    n = min(lens, max_len)
    k, v = _kv(("ends", B, Lq), B, 64, Hkv, dh)
    cache = _cache(B, Hkv, 64, dh, 255)
    vb.vla_op_kv4_store(ref.to_dev(k), ref.to_dev(v), None, _i32(*[n] * B), cache, 64)
    q = ref.normal(("endsq", B, Lq), (B, Lq, H, dh))
    got = _attend(ref.to_dev(q), cache, 64, Hkv, [lens] * B, max_len)
    if n == 0:
        assert (got == 0).all()
    else:
        _check(got, q, k[:, :n], v[:, :n], [n] * B, 0, 0)
