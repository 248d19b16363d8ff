"""The 8-bit KV cache and the attention over it, against float64."""
import numpy as np
import pytest

import kv8_ref as ref

pytestmark = pytest.mark.gpu


def _vb():
    from paper_2608_14586_amd import binding
    return binding


def _cache(B, Hkv, L_cap, dh, byte=0):
    import torch
    return torch.full((_vb().vla_op_kv8_bytes(B, Hkv, L_cap, dh),), byte, dtype=torch.uint8, device="cuda")


def _i32(*v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _kv(tag, B, L, Hkv, dh):
    k, v = (ref.normal((n,) + tag, (B, L, Hkv, dh)) for n in "kv")
    return ref.bf16(k * (1 + 4 * (np.arange(dh) % 23 == 0))), v  # a few strong channels


def _load(cache, L_cap, B, L, Hkv, dh, start=None, count=None, fill=0.0):
    import torch
    k = torch.full((B, L, Hkv, dh), fill, dtype=torch.bfloat16, device="cuda")
    v = torch.full((B, L, Hkv, dh), fill, dtype=torch.bfloat16, device="cuda")
    _vb().vla_op_kv8_load(cache, L_cap, start, count, k, v)
    return ref.from_dev(k), ref.from_dev(v)


def _same(a, b):
    with np.errstate(all="ignore"):
        return np.array_equal(a, np.asarray(b, np.float32), equal_nan=True)


def test_every_bf16_value():
    """All 65536 bf16 numbers, each in blocks of several exponents: codes to the last bit, NaN for what is not finite."""
    dh, L = 128, 512
    x = np.arange(65536, dtype=np.uint32).astype(np.uint32) << 16
    x = x.view(np.float32).reshape(1, L, 1, dh)
    order = np.random.default_rng(3).permutation(65536)
    mixed = x.reshape(-1)[order].reshape(x.shape)
    for a in (x, mixed, np.where(np.abs(mixed) < 500, mixed, 1.0).astype(np.float32)):
        cache = _cache(1, 1, L, dh)
        _vb().vla_op_kv8_store(ref.to_dev(a), ref.to_dev(a[:, ::-1]), None, None, cache, L)
        got = _load(cache, L, 1, L, 1, dh)
        for y, g in ((a[0], got[0][0]), (a[0, ::-1], got[1][0])):
            c = ref.Cache(L, 1, dh)
            c.store(y, 0)
            assert _same(g, c.values())


@pytest.mark.parametrize("B,L,Hkv,dh,start", [(1, 1, 1, 64, 0), (1, 1, 1, 128, 31), (2, 33, 2, 64, 5), (1, 64, 3, 128, 0),
                                              (3, 40, 1, 128, 63), (2, 200, 4, 64, 17), (1, 31, 8, 128, 32)])
def test_store_and_load(B, L, Hkv, dh, start):
    """Rows behind earlier ones, smaller and larger than those: exponents grow and the block's earlier codes follow; other
    blocks stay, and so does what another sequence holds."""
    L_cap = (start + 1 + L + 31) // 32 * 32
    old_k, old_v = _kv(("old", B, L, dh), B, L_cap, Hkv, dh)
    k, v = _kv((B, L, Hkv, dh), B, L, Hkv, dh)
    grow = np.exp2(np.arange(B * Hkv) * 3 - 5.0).reshape(B, 1, Hkv, 1)
    k, v = ref.bf16(k * grow), ref.bf16(v / grow)
    cache = _cache(B, Hkv, L_cap, dh, 0x5a)
    want = [[ref.Cache(L_cap, Hkv, dh) for _ in range(B)] for _ in range(2)]
    starts = [start + b % 2 for b in range(B)]
    for a, c, at in (((old_k, old_v), L_cap, [0] * B), ((k, v), L, starts)):
        _vb().vla_op_kv8_store(ref.to_dev(a[0]), ref.to_dev(a[1]), _i32(*at), None, cache, L_cap)
        for p in range(2):
            for b in range(B):
                want[p][b].store(a[p][b], at[b])
    got = _load(cache, L_cap, B, L_cap, Hkv, dh)
    for p in range(2):
        for b in range(B):
            assert _same(got[p][b], want[p][b].values())
    part = _load(cache, L_cap, B, L, Hkv, dh, _i32(*starts))
    assert all(_same(part[p][b], want[p][b].values()[starts[b]:starts[b] + L]) for p in range(2) for b in range(B))


def test_tokens_one_by_one():
    """Appending, with growing and shrinking magnitudes, and starting a used slot again from position 0."""
    B, L, Hkv, dh, L_cap = 2, 70, 2, 128, 96
    k, v = _kv(("one",), B, L, Hkv, dh)
    size = np.exp2(np.random.default_rng(1).integers(-12, 12, (B, L, Hkv, 1)).astype(np.float64))
    k, v = ref.bf16(k * size), ref.bf16(v * size[:, ::-1])
    cache = _cache(B, Hkv, L_cap, dh)
    for again in range(2):
        want = [[ref.Cache(L_cap, Hkv, dh) for _ in range(B)] for _ in range(2)]
        at = 0
        for n in ([1] * L, [5, 1, 31, 33])[again]:
            _vb().vla_op_kv8_store(ref.to_dev(k[:, at:at + n]), ref.to_dev(v[:, at:at + n]), _i32(at, at), None, cache, L_cap)
            for b in range(B):
                want[0][b].store(k[b, at:at + n], at)
                want[1][b].store(v[b, at:at + n], at)
            at += n
        assert at == L
        got = _load(cache, L_cap, B, L, Hkv, dh)
        for p in range(2):
            for b in range(B):
                assert _same(got[p][b], want[p][b].values()[:L]), again
        k, v = ref.bf16(k * 2.0 ** -20), ref.bf16(v * 2.0 ** -20)  # far smaller: the old exponents would leave zeros


def test_store_bounds_counts_and_strides():
    """Positions outside the cache and tokens past a sequence's count are left out, in both directions; heads before
    tokens, rows of a fused projection."""
    import torch
    B, L, Hkv, dh, L_cap = 7, 50, 2, 64, 64
    k, v = _kv(("bounds",), B, L, Hkv, dh)
    zero_k, zero_v = _kv(("before",), B, L_cap, Hkv, dh)
    start = [-20, 40, 64, -60, 10, 2 ** 31 - 1, -2 ** 31]
    count = [L, L, L, L, 0, L, 999]
    cache = _cache(B, Hkv, L_cap, dh, 17)
    _vb().vla_op_kv8_store(ref.to_dev(zero_k), ref.to_dev(zero_v), None, None, cache, L_cap)
    rows = torch.zeros((B, L, 5 * Hkv, dh), dtype=torch.bfloat16, device="cuda")
    rows[:, :, 2 * Hkv:3 * Hkv] = ref.to_dev(k)
    vh = ref.to_dev(v).transpose(1, 2).contiguous()  # [B][Hkv][L][dh]
    _vb().vla_op_kv8_store(rows[:, :, 2 * Hkv:3 * Hkv], vh.transpose(1, 2), _i32(*start), _i32(*count), cache, L_cap)
    after = _load(cache, L_cap, B, L_cap, Hkv, dh)
    got = _load(cache, L_cap, B, L, Hkv, dh, _i32(*start), _i32(*count), fill=3.0)
    for p, (old, x) in enumerate(((zero_k, k), (zero_v, v))):
        for b in range(B):
            c = ref.Cache(L_cap, Hkv, dh)
            c.store(old[b], 0)
            c.store(x[b], start[b], count[b])
            assert _same(after[p][b], c.values())
            for t in range(L):
                there = t < min(max(count[b], 0), L) and 0 <= start[b] + t < L_cap
                assert _same(got[p][b, t], c.values()[start[b] + t] if there else np.full((Hkv, dh), 3.0))


def test_far_offsets():
    """A cache past 4 GiB: the last head's last blocks."""
    import torch
    B, Hkv, dh, L_cap = 1, 18, 128, 1 << 20
    cache = torch.empty(_vb().vla_op_kv8_bytes(B, Hkv, L_cap, dh), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    L = 40
    k, v = _kv(("far",), B, L, Hkv, dh)
    start = L_cap - 64
    _vb().vla_op_kv8_store(ref.to_dev(k), ref.to_dev(v), _i32(start), None, cache, L_cap)
    got = _load(cache, L_cap, B, L, Hkv, dh, _i32(start))
    q = ref.normal(("farq",), (1, 1, 2 * Hkv, dh))
    n, window = start + L, L
    o = torch.empty((1, 1, 2 * Hkv, dh), dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(_vb().vla_op_attention_kv8_scratch(1, 1, 2 * Hkv, Hkv, dh, L_cap, window) + 16, dtype=torch.uint8, device="cuda")
    _vb().vla_op_attention_kv8(ref.to_dev(q), cache, L_cap, Hkv, _i32(n), o, L_cap, window, 0, scratch)
    want = []
    for p, x in ((0, k), (1, v)):
        c = ref.Cache(64, Hkv, dh)
        c.store(x[0], 0)
        assert _same(got[p][0], c.values()[:L])
        want.append(c.values())
    r, tol = ref.attention(q[0], want[0], want[1], L)
    assert np.all(np.abs(ref.from_dev(o)[0] - r) <= tol)


# -------------------------------------------------------------------- attention

def _attend(q, cache, L_cap, Hkv, lens, max_len, window=0, sinks=0, fill=9.0, extra=0):
    import torch
    B, Lq, H, dh = q.shape
    o = torch.full((B, Lq, H, dh), fill, dtype=torch.bfloat16, device="cuda")
    n = _vb().vla_op_attention_kv8_scratch(B, Lq, H, Hkv, dh, max_len, window, sinks)
    scratch = torch.full((n + extra,), 0x7f, dtype=torch.uint8, device="cuda") if n + extra else None
    _vb().vla_op_attention_kv8(ref.to_dev(q), cache, L_cap, Hkv, _i32(*lens), o, max_len, window, sinks, scratch)
    return ref.from_dev(o)


def _filled(k, v, L_cap, lens, byte=0x7f):
    """A cache with those rows, NaN codes (byte 0x7f) wherever nothing was stored; and the values it holds."""
    B, L, Hkv, dh = k.shape
    cache = _cache(B, Hkv, L_cap, dh, byte)
    _vb().vla_op_kv8_store(ref.to_dev(k), ref.to_dev(v), None, _i32(*lens), cache, L_cap)
    held = []
    for x in (k, v):
        rows = []
        for b in range(B):
            c = ref.Cache(L_cap, Hkv, dh)
            c.store(ref.bf16(x[b]), 0, lens[b])  # what the device gets
            rows.append(c.values())
        held.append(rows)
    return cache, held


def _check(o, q, held, lens, window=0, sinks=0):
    for b, n in enumerate(lens):
        r, tol = ref.attention(q[b], held[0][b], held[1][b], n, window, sinks)
        assert np.all(np.abs(o[b] - r) <= tol), (b, n, float(np.nanmax(np.abs(o[b] - r) / tol)))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv,Lq", [(1, 1, 1), (8, 8, 1), (14, 2, 1), (32, 8, 1), (8, 1, 3), (16, 1, 1), (20, 1, 1), (6, 2, 8), (28, 4, 5)])
def test_attention(dh, H, Hkv, Lq):
    lens = [1, 31, 32, 33, 64, 100, 257, 700]
    L_cap, L = 704, 700
    k, v = _kv(("att", H, Lq, dh), len(lens), L, Hkv, dh)
    q = ref.normal(("attq", H, Lq, dh), (len(lens), Lq, H, dh))
    cache, held = _filled(k, v, L_cap, lens)
    for max_len in (700, 704):
        _check(_attend(q, cache, L_cap, Hkv, lens, max_len), q, held, lens)


@pytest.mark.parametrize("dh,B,H,Hkv,Lq,lens,window,sinks", [
    (64, 1, 21, 3, 16, [6001], 0, 0), (128, 3, 14, 1, 9, [4100, 9, 2500], 0, 0), (64, 2, 40, 1, 7, [3333, 0], 0, 0),
    (128, 1, 5, 5, 40, [3000], 0, 0), (64, 1, 21, 3, 16, [6001], 1500, 40), (128, 9, 16, 1, 2, [700, 1, 2900, 33, 64, 1500, 2, 0, 2222], 0, 0)])
def test_attention_tiles_and_splits(dh, B, H, Hkv, Lq, lens, window, sinks):
    """Several tiles of queries over keys that several workgroups share, their numbers no multiples of eight."""
    L = max(lens)
    L_cap = (L + 31) // 32 * 32
    k, v = _kv(("tiles", H, Lq, dh), B, L, Hkv, dh)
    q = ref.normal(("tilesq", H, Lq, dh), (B, Lq, H, dh))
    cache, held = _filled(k, v, L_cap, lens)
    assert _vb().vla_op_attention_kv8_scratch(B, Lq, H, Hkv, dh, L, window, sinks) > 0
    o = _attend(q, cache, L_cap, Hkv, lens, L, window, sinks)
    _check(o, q, held, lens, window, sinks)
    assert np.array_equal(o, _attend(q, cache, L_cap, Hkv, lens, L, window, sinks))


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (32, 4), (33, 40), (100, 1), (250, 16), (699, 3), (5000, 2)])
def test_attention_window(window, sinks):
    lens = [3, 40, 333, 600]
    L_cap = 608
    for Lq, H, Hkv in ((1, 4, 2), (4, 8, 1), (7, 6, 2)):
        k, v = _kv(("win", window, Lq), 4, 600, Hkv, 64)
        q = ref.normal(("winq", window, Lq), (4, Lq, H, 64))
        cache, held = _filled(k, v, L_cap, lens)
        _check(_attend(q, cache, L_cap, Hkv, lens, 600, window, sinks), q, held, lens, window, sinks)


def test_attention_long_and_split():
    for B, H, Hkv, dh, n in ((1, 8, 2, 128, 30000), (2, 4, 4, 64, 9001)):
        lens = [n] + [n // 3] * (B - 1)
        L_cap = (n + 31) // 32 * 32
        k, v = _kv(("long", n), B, n, Hkv, dh)
        q = ref.normal(("longq", n), (B, 1, H, dh), 3.0)
        cache, held = _filled(k, v, L_cap, lens)
        assert _vb().vla_op_attention_kv8_scratch(B, 1, H, Hkv, dh, n) > 0
        _check(_attend(q, cache, L_cap, Hkv, lens, n), q, held, lens)


def test_lengths_that_leave_nothing_and_cut_ones():
    """Length 0, fewer tokens than queries (rows that see no key are zeros), lengths below zero and above max_len."""
    lens, Lq, H, Hkv, dh, L_cap = [0, 2, -5, 100], 4, 4, 2, 64, 64
    k, v = _kv(("none",), 4, 64, Hkv, dh)
    q = ref.normal(("noneq",), (4, Lq, H, dh))
    cache, held = _filled(k, v, L_cap, [64] * 4)
    o = _attend(q, cache, L_cap, Hkv, lens, 50)
    assert not o[0].any() and not o[2].any() and not o[1, :2].any()
    _check(o, q, held, [0, 2, 0, 50])


def test_values_that_are_not_finite():
    """NaN keys and values: queries that see them get NaN (in that dim for a value), others are as without them; what no query sees may be NaN."""
    B, L, H, Hkv, dh, Lq, L_cap = 1, 100, 4, 1, 64, 6, 128
    k, v = _kv(("nan",), B, L, Hkv, dh)
    q = ref.normal(("nanq",), (B, Lq, H, dh))
    for window, sinks in ((0, 0), (20, 3)):
        for where in (97, 96, 99, 78, 1, 2, 50, 77):
            for part in ("k", "v"):
                kk, vv = k.copy(), v.copy()
                (kk if part == "k" else vv)[0, where, 0, 7] = [np.nan, np.inf, -np.inf][where % 3]
                clean, held = _filled(k, v, L_cap, [L])
                cache, _ = _filled(kk, vv, L_cap, [L])
                base = _attend(q, clean, L_cap, Hkv, [L], L, window, sinks)
                o = _attend(q, cache, L_cap, Hkv, [L], L, window, sinks)
                for i in range(Lq):
                    p = L - Lq + i
                    sees = where <= p and (not window or p - where < window or where < sinks)
                    hit = np.isnan(o[0, i])
                    if part == "k":
                        assert hit.all() if sees else not hit.any(), (window, where, i)
                    else:
                        assert (hit[:, 7].all() if sees else not hit.any()) and not np.delete(hit, 7, 1).any(), (window, where, i)
                assert not np.isnan(base).any()
                # queries that do not see it: as if it were not there (its block's exponent is that of the finite ones)
                alter = kk if part == "k" else vv
                c = ref.Cache(L_cap, Hkv, dh)
                c.store(np.where(np.isfinite(alter[0]), alter[0], np.nan), 0)
                h2 = [c.values(), held[1][0]] if part == "k" else [held[0][0], c.values()]
                h2 = [np.nan_to_num(x, nan=0.0) for x in h2]
                for i in range(Lq):
                    p = L - Lq + i
                    sees = where <= p and (not window or p - where < window or where < sinks)
                    if not sees:
                        r2, t2 = ref.attention(q[0], h2[0], h2[1], L, window, sinks)
                        assert np.all(np.abs(o[0, i] - r2[i]) <= t2[i])


def test_magnitudes():
    """Blocks of very different sizes side by side; the largest numbers; queries that are not finite stay in their rows."""
    B, L, H, Hkv, dh, L_cap = 1, 200, 8, 2, 128, 224
    k, v = _kv(("mag",), B, L, Hkv, dh)
    v = ref.bf16(v * np.exp2((np.arange(L) // 32 * 12 - 40.0)).reshape(1, L, 1, 1))
    q = ref.normal(("magq",), (B, 2, H, dh))
    cache, held = _filled(k, v, L_cap, [L])
    _check(_attend(q, cache, L_cap, Hkv, [L], L), q, held, [L])
    v2 = ref.bf16(np.sign(v) * np.where(np.abs(v) > 0, 3e38, 0))
    cache, held = _filled(k, v2, L_cap, [L])
    o = _attend(q, cache, L_cap, Hkv, [L], L)
    assert np.isfinite(o).all()
    _check(o, q, held, [L])
    bad = q.copy()
    bad[0, 1, 3, 5] = np.nan
    bad[0, 0, 2, 0] = np.inf
    cache, held = _filled(k, v, L_cap, [L])
    o, base = _attend(bad, cache, L_cap, Hkv, [L], L), _attend(q, cache, L_cap, Hkv, [L], L)
    assert np.isnan(o[0, 1, 3]).all() and np.isnan(o[0, 0, 2]).all()
    keep = np.ones((2, H), bool)
    keep[1, 3] = keep[0, 2] = False
    assert np.array_equal(o[0][keep], base[0][keep])


def test_large_scores_one_key_each():
    """Scores hundreds apart: the maximum moves block by block, and one key takes all the weight."""
    L, H, Hkv, dh, L_cap = 320, 4, 4, 64, 320
    k, v = _kv(("peak",), 1, L, Hkv, dh)
    k = ref.bf16(k * 0.01)
    for h in range(Hkv):
        k[0, :, h, 0] = np.linspace(-400, 400, L) if h % 2 else np.linspace(400, -400, L)
    q = ref.normal(("peakq",), (1, 1, H, dh))
    q[..., 0] = 8
    cache, held = _filled(k, v, L_cap, [L])
    _check(_attend(q, cache, L_cap, Hkv, [L], L), q, held, [L])


def test_calls_repeat_their_bits():
    lens = [100, 700, 350]
    k, v = _kv(("bits",), 3, 700, 2, 128)
    q = ref.normal(("bitsq",), (3, 1, 8, 128))
    cache, _ = _filled(k, v, 704, lens)
    a, b = _attend(q, cache, 704, 2, lens, 700), _attend(q, cache, 704, 2, lens, 700, extra=64)
    assert np.array_equal(a, b)


def test_scratch_never_falls_with_the_length():
    for B, H, Hkv, dh in ((1, 8, 1, 128), (3, 32, 8, 64)):
        last = 0
        for n in list(range(1, 3000, 37)) + [10000, 100000, 1 << 20]:
            s = _vb().vla_op_attention_kv8_scratch(B, 1, H, Hkv, dh, n)
            assert s >= last
            last = s


def test_graph_with_growing_lengths():
    """Store and attention of a decode step in a graph, replayed for one token after another."""
    import torch
    vb = _vb()
    B, H, Hkv, dh, L_cap, n0, steps = 2, 8, 2, 128, 160, 60, 5
    k, v = _kv(("graph",), B, n0 + steps, Hkv, dh)
    q = ref.normal(("graphq",), (steps, B, 1, H, dh))
    cache, _ = _filled(k[:, :n0], v[:, :n0], L_cap, [n0] * B)
    dk, dv = (torch.empty((B, 1, Hkv, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dq, o = (torch.empty((B, 1, H, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at, lens = _i32(0, 0), _i32(0, 0)
    scratch = torch.empty(vb.vla_op_attention_kv8_scratch(B, 1, H, Hkv, dh, L_cap) + 16, dtype=torch.uint8, device="cuda")

    def step():
        vb.vla_op_kv8_store(dk, dv, at, None, cache, L_cap)
        vb.vla_op_attention_kv8(dq, cache, L_cap, Hkv, lens, o, L_cap, scratch=scratch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    want = [[ref.Cache(L_cap, Hkv, dh) for _ in range(B)] for _ in range(2)]
    for b in range(B):
        want[0][b].store(k[b, :n0], 0)
        want[1][b].store(v[b, :n0], 0)
    for s in range(steps):
        n = n0 + s
        dk.copy_(ref.to_dev(k[:, n:n + 1])), dv.copy_(ref.to_dev(v[:, n:n + 1])), dq.copy_(ref.to_dev(q[s]))
        at.fill_(n), lens.fill_(n + 1)
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            want[0][b].store(k[b, n:n + 1], n)
            want[1][b].store(v[b, n:n + 1], n)
        _check(ref.from_dev(o), q[s], [[c.values() for c in p] for p in want], [n + 1] * B)
