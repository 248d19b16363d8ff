"""A decoder block in 8 bits over packed prompts, and its decode steps over the 8-bit
cache: every call's result against 64 bits from the inputs that the run gave it, with the bounds
of the operators' own tests; then the run in a graph and on two streams at once.

Rows of codes: half a step, scale / 2, and 80 2^-24 of the value for fp32 sums.  Rotated heads: fp32
throughout (2^-18 of the pair's sizes) and a bf16 result."""
import numpy as np
import pytest

import kv8_ref as ref
from test_gpu_i8 import _cuda, _pack, _ref_gemm, _rng
from test_gpu_packed import _reference as _packed_attention

pytestmark = pytest.mark.gpu
EPS = 1e-6
U32, UB = 2.0 ** -24, 2.0 ** -8
SIZES = [dict(d=256, H=4, Hkv=2, dh=64, F=512), dict(d=384, H=3, Hkv=3, dh=128, F=320)]


def _np(t):
    return t.double().cpu().numpy()


class _Block:
    """Weights and tables; run() is the whole block over rows in place of h."""

    def __init__(self, d, H, Hkv, dh, F, cap=96):
        import torch
        from paper_2608_14586_amd import binding as vb
        self.vb, self.d, self.H, self.Hkv, self.dh, self.F, self.cap = vb, d, H, Hkv, dh, F, cap
        self.N = (H + 2 * Hkv) * dh
        rng = _rng(71, d, dh)

        def weights(N, K):
            w = rng.integers(-127, 128, (N, K), dtype=np.int8)
            s = (rng.uniform(0.5, 1.5, N) / (73 * np.sqrt(K))).astype(np.float32)
            return w, s, _pack(w, s)

        self.qkv, self.o, self.gu, self.down = weights(self.N, d), weights(d, H * dh), weights(2 * F, d), weights(d, F)
        self.g1, self.g2 = (_cuda(rng.uniform(0.5, 1.5, d).astype(np.float32)) for _ in range(2))
        self.gq, self.gk = (_cuda(rng.uniform(0.5, 1.5, dh).astype(np.float32)) for _ in range(2))
        ang = np.arange(cap)[:, None] * 10000.0 ** (-np.arange(0, dh, 2) / dh)
        self.cos, self.sin = (_cuda(f(ang).astype(np.float32)) for f in (np.cos, np.sin))
        torch.cuda.synchronize()

    def buffers(self, T, B, Lq):
        import torch
        new = lambda dt, *s: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
        i8, bf, f32 = torch.int8, torch.bfloat16, torch.float32
        n = self.vb.vla_op_attention_kv8_scratch(B, Lq, self.H, self.Hkv, self.dh, self.cap)
        return dict(c1=new(i8, T, self.d), s1=new(f32, T), qkv=new(bf, T, self.N), q=new(bf, T, self.H, self.dh),
                    k=new(bf, T, self.Hkv, self.dh), o=new(bf, T, self.H, self.dh), c2=new(i8, T, self.H * self.dh),
                    s2=new(f32, T), y=new(bf, T, self.d), c3=new(i8, T, self.d), s3=new(f32, T), a=new(bf, T, self.F),
                    c4=new(i8, T, self.F), s4=new(f32, T), h1=new(f32, T, self.d),
                    scratch=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))

    def run(self, h, h_out, b, pos, cache, attend):
        """h [T][d] fp32 -> h_out; b: buffers; attend(q, k, v): the cache's part and the attention."""
        vb, T, H, Hkv, dh = self.vb, len(h), self.H, self.Hkv, self.dh
        vb.vla_op_norm_i8(h, None, None, self.g1, EPS, b["c1"], b["s1"])
        vb.vla_op_gemm_i8(b["c1"], b["s1"], self.qkv[2], None, b["qkv"], self.N)
        rows = b["qkv"].view(1, T, H + 2 * Hkv, dh)
        vb.vla_op_qk_norm_rope(rows[:, :, :H], rows[:, :, H:H + Hkv], self.gq, self.gk, EPS, self.cos, self.sin, pos.view(1, T),
                               b["q"].view(1, T, H, dh), b["k"].view(1, T, Hkv, dh))
        attend(b["q"], b["k"], rows[0, :, H + Hkv:])
        vb.vla_op_norm_i8(b["o"].view(T, H * dh), None, None, None, 0.0, b["c2"], b["s2"])
        vb.vla_op_gemm_i8(b["c2"], b["s2"], self.o[2], None, b["y"], self.d)
        vb.vla_op_norm_i8(h, b["y"], b["h1"], self.g2, EPS, b["c3"], b["s3"])
        vb.vla_op_gemm_i8(b["c3"], b["s3"], self.gu[2], None, b["a"], 2 * self.F, True)
        vb.vla_op_norm_i8(b["a"], None, None, None, 0.0, b["c4"], b["s4"])
        h_out.copy_(b["h1"])
        vb.vla_op_gemm_i8(b["c4"], b["s4"], self.down[2], h_out, h_out, self.d)

    def prefill(self, h, h_out, b, offsets, pos, cache):
        vb, B, T = self.vb, len(offsets) - 1, len(h)
        start, count = -offsets[:-1], offsets[1:]  # prompt i's rows begin behind offsets[i] others

        def attend(q, k, v):
            each = lambda x: x.unsqueeze(0).expand(B, T, self.Hkv, self.dh)  # noqa: E731
            vb.vla_op_kv8_store(each(k), each(v), start, count, cache, self.cap)
            vb.vla_op_attention_packed(q, k, v, offsets, b["o"])
        self.run(h, h_out, b, pos, cache, attend)

    def step(self, h, h_out, b, lens, cache):
        """A token for each sequence, of lens tokens so far."""
        vb, B = self.vb, len(h)

        def attend(q, k, v):
            vb.vla_op_kv8_store(k.view(B, 1, self.Hkv, self.dh), v.unsqueeze(1), lens, None, cache, self.cap)
            vb.vla_op_attention_kv8(q.view(B, 1, self.H, self.dh), cache, self.cap, self.Hkv, lens + 1,
                                    b["o"].view(B, 1, self.H, self.dh), self.cap, 0, 0, b["scratch"])
        self.run(h, h_out, b, lens, cache, attend)

    # ---------------------------------------------------------------- checks in 64 bits
    def check(self, h, h_out, b, pos):
        H, Hkv, dh = self.H, self.Hkv, self.dh

        def close(got, want, tol, what):
            got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
            assert np.all(np.abs(got - want) <= tol), (what, np.max(np.abs(got - want) / np.maximum(tol, 1e-300)))

        def codes(c, s, t, g, what):
            t = t.astype(np.float64)
            v = t if g is None else t * _np(g) / np.sqrt((t ** 2).mean(-1, keepdims=True) + EPS)
            s = _np(s)[:, None]
            close(_np(c) * s, v, s / 2 + np.abs(v).max(-1, keepdims=True) * 80 * U32, what)

        def product(c, s, w, got, what, residual=None, gated=False):
            y = _ref_gemm(c.cpu().numpy(), s.cpu().numpy(), w[0], w[1], gated)
            if residual is not None:
                close(got, y + residual, (np.abs(y) + np.abs(y + residual)) * 4 * U32, what)
            else:
                close(got, y, np.abs(y) * (UB + (2.0 ** -17 if gated else 4 * U32)) + 1e-37, what)

        codes(b["c1"], b["s1"], _np(h), self.g1, "first norm")
        product(b["c1"], b["s1"], self.qkv, _np(b["qkv"]), "qkv")
        rows = _np(b["qkv"]).reshape(len(h), H + 2 * Hkv, dh)
        at = pos.cpu().numpy()
        cos, sin = _np(self.cos)[at][:, None], _np(self.sin)[at][:, None]
        for x, g, got, what in ((rows[:, :H], self.gq, b["q"], "q"), (rows[:, H:H + Hkv], self.gk, b["k"], "k")):
            y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + EPS) * _np(g)
            lo, hi = y[..., :dh // 2], y[..., dh // 2:]
            want = np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], -1)
            size = np.concatenate([np.abs(lo) + np.abs(hi)] * 2, -1)
            close(_np(got), want, np.abs(want) * UB + size * 2.0 ** -18, what)
        codes(b["c2"], b["s2"], _np(b["o"]).reshape(len(h), -1), None, "attention's rows")
        product(b["c2"], b["s2"], self.o, _np(b["y"]), "output projection")
        assert bool((b["h1"] == h + b["y"].float()).all())
        codes(b["c3"], b["s3"], _np(b["h1"]), self.g2, "second norm")
        product(b["c3"], b["s3"], self.gu, _np(b["a"]), "gate and up", gated=True)
        codes(b["c4"], b["s4"], _np(b["a"]), None, "gated rows")
        product(b["c4"], b["s4"], self.down, _np(h_out), "down", residual=_np(b["h1"]))
        return rows[:, H + Hkv:]


def _hidden(key, T, d):
    return _cuda(_rng(72, key).standard_normal((T, d)).astype(np.float32))


def _i32(v):
    return _cuda(np.asarray(v, np.int32))


def _positions(offsets, T):
    pos = np.zeros(T, np.int32)
    for a, b in zip(offsets, offsets[1:]):
        pos[a:b] = np.arange(b - a)
    return pos


def _cache_of(block, B):
    import torch
    return torch.zeros(block.vb.vla_op_kv8_bytes(B, block.Hkv, block.cap, block.dh), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("size", SIZES, ids=["grouped", "wide"])
@pytest.mark.parametrize("lens", [[40, 1, 0, 33], [7], [1, 1, 1], [64, 90, 31, 32, 5]], ids=str)
def test_prompts_and_steps(size, lens):
    import torch
    blk = _Block(**size)
    B, at = len(lens), np.concatenate([[0], np.cumsum(lens)])
    T = int(at[-1])
    h, h_out = _hidden(T, T, blk.d), torch.zeros((T, blk.d), device="cuda")
    b, cache, pos = blk.buffers(T, B, 1), _cache_of(blk, B), _i32(_positions(at, T))
    blk.prefill(h, h_out, b, _i32(at), pos, cache)
    v = blk.check(h, h_out, b, pos)
    q, k = _np(b["q"]), _np(b["k"])
    o, tol = _packed_attention(q, k, v, list(at))
    assert np.all(np.abs(_np(b["o"]) - o) <= tol)
    keys, values = ([ref.Cache(blk.cap, blk.Hkv, blk.dh) for _ in lens] for _ in range(2))
    for i in range(B):
        keys[i].store(k[at[i]:at[i + 1]], 0)
        values[i].store(v[at[i]:at[i + 1]], 0)

    def same_cache():
        back = [torch.zeros((B, blk.cap, blk.Hkv, blk.dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        blk.vb.vla_op_kv8_load(cache, blk.cap, None, None, *back)
        for i in range(B):
            for got, want in zip(back, (keys, values)):
                assert np.array_equal(_np(got[i])[:now[i]], want[i].values()[:now[i]]), i

    now = list(lens)
    same_cache()
    sb = blk.buffers(B, B, 1)
    for t in range(3):
        h, h_out = _hidden(100 * t + B, B, blk.d), torch.zeros((B, blk.d), device="cuda")
        n = _i32(now)
        blk.step(h, h_out, sb, n, cache)
        v = blk.check(h, h_out, sb, n)
        q, k = _np(sb["q"]), _np(sb["k"])
        for i in range(B):
            keys[i].store(k[i:i + 1], now[i])
            values[i].store(v[i:i + 1], now[i])
            now[i] += 1
            o, tol = ref.attention(q[i:i + 1], keys[i].values(), values[i].values(), now[i])
            assert np.all(np.abs(_np(sb["o"][i:i + 1]) - o) <= tol), (t, i)
        same_cache()


def _everything(blk, h, at, pos, hs, n, mine):
    blk.prefill(h, mine["out"], mine["b"], at, pos, mine["cache"])
    blk.step(hs, mine["outs"], mine["bs"], n, mine["cache"])


def _own(blk, T, B):
    import torch
    return dict(out=torch.zeros((T, blk.d), device="cuda"), outs=torch.zeros((B, blk.d), device="cuda"),
                b=blk.buffers(T, B, 1), bs=blk.buffers(B, B, 1), cache=_cache_of(blk, B))


def test_in_a_graph():
    """Prompts of other lengths and other rows between the replays, each against the eager run."""
    import torch
    blk, T, B = _Block(**SIZES[0]), 100, 4
    ats = [[0, 40, 41, 41, 100], [0, 1, 2, 3, 4], [0, 70, 70, 90, 100], [3, 10, 40, 60, 99]]
    mine, eager = _own(blk, T, B), _own(blk, T, B)
    h, at, pos, hs, n = _hidden(0, T, blk.d), _i32(ats[0]), _i32(_positions(ats[0], T)), _hidden(1, B, blk.d), _i32(np.diff(ats[0]))
    _everything(blk, h, at, pos, hs, n, mine)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _everything(blk, h, at, pos, hs, n, mine)
    for i, a in enumerate(ats + ats[:1]):
        h.copy_(_hidden(10 + i, T, blk.d))
        hs.copy_(_hidden(20 + i, B, blk.d))
        at.copy_(_i32(a))
        pos.copy_(_i32(_positions(a, T)))
        n.copy_(_i32(np.diff(a)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _everything(blk, h, at, pos, hs, n, eager)
        torch.cuda.synchronize()
        rows = slice(a[0], a[-1])  # rows in no prompt keep the attention's old ones
        assert torch.equal(mine["out"][rows], eager["out"][rows]) and torch.equal(mine["outs"], eager["outs"]), i
        for x in ("o", "qkv", "k"):
            assert torch.equal(mine["b"][x][rows], eager["b"][x][rows]), (i, x)


def test_two_at_once():
    """Two streams, memory of their own, one set of weights; each has the results that it has alone."""
    import torch
    blk, B = _Block(**SIZES[1]), 3
    jobs = []
    for i, a in enumerate(([0, 50, 120, 130], [0, 3, 90, 150])):
        T = a[-1]
        jobs.append((_hidden(30 + i, T, blk.d), _i32(a), _i32(_positions(a, T)), _hidden(40 + i, B, blk.d), _i32(np.diff(a))))
    alone = [_own(blk, len(j[0]), B) for j in jobs]
    for j, m in zip(jobs, alone):
        _everything(blk, *j, m)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    both = [_own(blk, len(j[0]), B) for j in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        for j, m, s in zip(jobs, both, streams):
            with torch.cuda.stream(s):
                _everything(blk, *j, m)
    for s in streams:
        s.synchronize()
    for m, w in zip(both, alone):
        assert torch.equal(m["out"], w["out"]) and torch.equal(m["outs"], w["outs"])
        assert torch.equal(m["cache"], w["cache"])
