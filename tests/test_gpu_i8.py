"""Rows into int8 codes, and products of int8 rows with int8 weights, against 64 bits.

Codes are compared as they are.  Scales: max|u| / 127 is two roundings (2^-24 each);
the norm's factor has a sum of d squares in fp32, at most 54 additions deep, a mean, a
root and a quotient: 64 * 2^-24.  Products: the sum of codes is exact; its conversion
and two factors are 3 * 2^-24, an addition 2^-24 of the result, a bf16 result 2^-8
half a step."""
import numpy as np
import pytest
import torch

from i8_tiles import TILES
from paper_2608_14586_amd import binding as vb

pytestmark = pytest.mark.gpu
U32, UB = 2.0 ** -24, 2.0 ** -8


def _rng(*key):
    return np.random.default_rng(list(key))


def _cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _strided(shape, dtype, pad, fill):
    """[M, n] whose rows lie n + pad apart, and the whole memory behind it."""
    whole = torch.full((shape[0], shape[1] + pad), fill, dtype=dtype, device="cuda")
    return whole[:, :shape[1]], whole


# ------------------------------------------------------------------- rows into codes

def _ref_norm(x, add, g, eps):
    t = x if add is None else x + add  # fp32, rounded once
    u = t if g is None else t * g
    top = np.abs(u).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        code = np.rint(127.0 * u.astype(np.float64) / top.astype(np.float64))
    scale = top[:, 0].astype(np.float64) / 127
    if g is not None:
        scale = scale / np.sqrt((t.astype(np.float64) ** 2).mean(-1) + np.float64(np.float32(eps)))
    return t, code, scale


@pytest.mark.parametrize("d", [8, 64, 504, 512, 520, 896, 1024, 1032, 2048, 4096, 4104, 8192, 11008, 12296, 16384, 16392, 32768])
@pytest.mark.parametrize("xt,at,norm", [("f32", None, True), ("f32", "bf16", True), ("bf16", None, False), ("f32", "f32", False)])
def test_norm_i8(d, xt, at, norm):
    rng = _rng(1, d, norm)
    M = 5
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    mk = lambda kind, s: _cuda(rng.standard_normal((M, d)) * s).to(dt[kind])
    x = mk(xt, 3.0)
    add = mk(at, 1.0) if at else None
    g = _cuda(rng.uniform(0.5, 1.5, d).astype(np.float32)) if norm else None
    xs, _ = _strided((M, d), dt[xt], 16, 7.0)
    xs.copy_(x)
    codes, whole = _strided((M, d), torch.int8, 24, 77)
    scales = torch.full((M + 1,), 5.0, device="cuda")
    total, tw = _strided((M, d), torch.float32, 8, 9.0)
    vb.vla_op_norm_i8(xs, add, total if at else None, g, 1e-6, codes, scales[:M])
    t, code, scale = _ref_norm(x.float().cpu().numpy(), None if add is None else add.float().cpu().numpy(),
                               None if g is None else g.cpu().numpy(), 1e-6)
    assert np.array_equal(codes.cpu().numpy(), code)
    assert np.all(np.abs(scales[:M].cpu().numpy() - scale) <= 64 * U32 * scale)
    assert scales[M] == 5.0 and bool((whole[:, d:] == 77).all())
    if at:
        assert np.array_equal(total.cpu().numpy(), t) and bool((tw[:, d:] == 9.0).all())


def test_norm_i8_borders():
    """Rows whose values lie on borders between codes (ties go to the even one), and an fp32 step beside them."""
    d = 512
    rows = []
    for top in (127.0, 254.0, 127.0 * 2 ** -60, 1.0, 3.0, 0.1, 1e30):
        top = np.float32(top)
        half = (np.arange(d) % 254 - 126.5) * np.float64(top) / 127
        v = half.astype(np.float32)
        v = np.where(np.arange(d) < 254, v, np.where(np.arange(d) % 2, np.nextafter(v, np.float32(np.inf)), np.nextafter(v, np.float32(-np.inf))))
        v[0] = top
        rows.append(np.clip(v, -top, top))
    x = np.stack(rows).astype(np.float32)
    codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(x), device="cuda")
    vb.vla_op_norm_i8(_cuda(x), None, None, None, 0.0, codes, scales)
    assert np.array_equal(codes.cpu().numpy(), _ref_norm(x, None, None, 0.0)[1])


def test_norm_i8_rows_that_are_not_finite_or_zero():
    M, d = 8, 896
    x = _rng(2).standard_normal((M, d)).astype(np.float32)
    x[0, 5], x[1, 895], x[2, 0] = np.nan, np.inf, -np.inf
    x[3] = 0
    x[4] *= np.float32(1e-32)
    x[5, 1:] = 0
    g = np.ones(d, np.float32)
    for gain in (None, g):
        for eps in (0.0, 1e-6):
            codes, scales = torch.empty((M, d), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
            vb.vla_op_norm_i8(_cuda(x), None, None, None if gain is None else _cuda(gain), eps, codes, scales)
            c, s = codes.cpu().numpy(), scales.cpu().numpy()
            assert np.isnan(s[:3]).all() and not c[:5].any() and (s[3:5] == 0).all()
            _, code, scale = _ref_norm(x[5:], None, gain, eps)
            assert np.array_equal(c[5:], code) and np.all(np.abs(s[5:] - scale) <= 64 * U32 * scale)


@pytest.mark.parametrize("d", [64, 1000, 4096, 11008, 32768])
@pytest.mark.parametrize("add", ["", "f32", "bf16", "into x", "into add"])
def test_norm_i8_rows_whose_squares_leave_fp32(d, add):
    rng = _rng(6, d)
    size = np.array([1e25, 1.0, 1e-25, 1e19, 3e-21, 1e37], np.float32)[:, None]
    x = rng.standard_normal((6, d)).astype(np.float32) * size / 8
    g = rng.uniform(0.5, 1.5, d).astype(np.float32)
    y = None if not add else (rng.standard_normal((6, d)).astype(np.float32) * size / 8)
    xd, yd = _cuda(x), None if y is None else _cuda(y)
    if add == "bf16":
        yd = yd.bfloat16()
        y = yd.float().cpu().numpy()
    total = {"into x": xd, "into add": yd}.get(add)
    codes, scales = torch.empty((6, d), dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    for eps in (0.0, 1e-6):
        if total is not None:
            xd.copy_(_cuda(x)), yd.copy_(_cuda(y))
        vb.vla_op_norm_i8(xd, yd, total, _cuda(g), eps, codes, scales)
        _, code, scale = _ref_norm(x, y, g, eps)
        assert np.array_equal(codes.cpu().numpy(), code)
        assert np.all(np.abs(scales.cpu().numpy() - scale) <= 64 * U32 * scale)


@pytest.mark.parametrize("xt,at", [("bf16", "f32"), ("bf16", "bf16"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("norm", [True, False])
def test_norm_i8_other_types(xt, at, norm):
    """Gain with bf16 rows, and a sum that is asked for where nothing is added."""
    rng = _rng(7, norm)
    M, d = 37, 1032
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = _cuda(rng.standard_normal((M, d)).astype(np.float32)).to(dt[xt])
    add = _cuda(rng.standard_normal((M, d)).astype(np.float32)).to(dt[at]) if at else None
    g = _cuda(rng.uniform(0.5, 1.5, d).astype(np.float32)) if norm else None
    codes, scales = torch.empty((M, d), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    total = torch.empty((M, d), device="cuda")
    vb.vla_op_norm_i8(x, add, total, g, 0.25, codes, scales)
    t, code, scale = _ref_norm(x.float().cpu().numpy(), None if add is None else add.float().cpu().numpy(),
                               None if g is None else g.cpu().numpy(), 0.25)
    assert np.array_equal(codes.cpu().numpy(), code) and np.array_equal(total.cpu().numpy(), t)
    assert np.all(np.abs(scales.cpu().numpy() - scale) <= 64 * U32 * scale)


def test_norm_i8_in_place():
    """The sum may go to x itself, or to add, and twice the same call gives the same bits."""
    rng = _rng(3)
    M, d = 33, 1000
    x, y = (_cuda(rng.standard_normal((M, d)).astype(np.float32)) for _ in range(2))
    g = _cuda(rng.uniform(0.5, 1.5, d).astype(np.float32))
    want = x + y
    for target in ("x", "add"):
        a, b = x.clone(), y.clone()
        codes, scales = torch.empty((M, d), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        vb.vla_op_norm_i8(a, b, a if target == "x" else b, g, 1e-6, codes, scales)
        assert torch.equal(a if target == "x" else b, want) and torch.equal(b if target == "x" else a, y if target == "x" else x)
        again, s2 = torch.empty_like(codes), torch.empty_like(scales)
        vb.vla_op_norm_i8(want, None, None, g, 1e-6, again, s2)
        assert torch.equal(codes, again) and torch.equal(scales, s2)


# --------------------------------------------------------------------- products

def _pack(w, sw):
    N, K = w.shape
    Wp = torch.empty(vb.vla_op_w8_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    vb.vla_op_w8_pack(_cuda(w), _cuda(sw), Wp)
    return Wp


def _ref_gemm(x, sx, w, sw, swiglu):
    y = (x.astype(np.float64) @ w.astype(np.float64).T) * sx.astype(np.float64)[:, None] * sw.astype(np.float64)
    if swiglu:
        h = y.shape[1] // 2
        g = y[:, :h]
        y = g / (1 + np.exp(-g)) * y[:, h:]
    return y


def _product(M, N, K, out, seed=0, wide=0):
    rng = _rng(4, M, N, K, seed)
    x = rng.integers(-128, 128, (M, K), dtype=np.int8)
    w = rng.integers(-128, 128, (N, K), dtype=np.int8)
    sx = rng.uniform(0.5, 2, M).astype(np.float32)
    sw = (rng.uniform(0.5, 2, N) / (5000 * np.sqrt(K))).astype(np.float32)
    swiglu = out == "swiglu"
    cols = N // 2 if swiglu else N
    xs, _ = _strided((M, K), torch.int8, 16 * (wide > 0), 99)
    xs.copy_(_cuda(x))
    dt = torch.float32 if out in ("f32", "add") else torch.bfloat16
    o, whole = _strided((M, cols), dt, wide, 3.0)
    res = None
    ref = _ref_gemm(x, sx, w, sw, swiglu)
    if out == "add":
        r = rng.standard_normal((M, cols)).astype(np.float32)
        o.copy_(_cuda(r))
        res = o
        ref = ref + r
        size = np.abs(ref) + np.abs(r)
    else:
        size = np.abs(ref)
    vb.vla_op_gemm_i8(xs, _cuda(sx), _pack(w, sw), res, o, N, swiglu)
    got = o.float().cpu().numpy().astype(np.float64)
    tol = size * (4 * U32 if dt == torch.float32 else UB + 4 * U32)
    if swiglu:  # e^-g by the hardware's exponential: |g| 2^-24 and 2^-22, g below 64 here
        tol = np.abs(ref) * (UB + 2.0 ** -17) + 1e-37
    assert np.all(np.abs(got - ref) <= tol), (M, N, K, out, np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)))
    assert bool((whole[:, cols:] == 3.0).all())


@pytest.mark.parametrize("M", [1, 2, 3, 15, 16, 17, 31, 33, 64, 65, 128, 130, 257])
@pytest.mark.parametrize("N,K", [(1, 16), (33, 48), (100, 272), (896, 896), (1027, 1040), (64, 4096)])
def test_gemm_i8(M, N, K):
    for out in ("bf16", "f32", "add"):
        _product(M, N, K, out, wide=4 if N % 4 == 0 else 3)


@pytest.mark.parametrize("M", [1, 7, 16, 40, 129, 300])
@pytest.mark.parametrize("N,K", [(64, 64), (192, 1024), (1792, 896), (9728, 144)])
def test_gemm_i8_gated(M, N, K):
    _product(M, N, K, "swiglu", wide=8)
    _product(M, N, K, "swiglu")


@pytest.mark.parametrize("tile", list(TILES))
def test_gemm_i8_tiles(tile):
    """Every tile at odd sizes, each output, aligned rows of outputs and others."""
    for M, N, K, gated in TILES[tile]:
        assert vb.vla_op_gemm_i8_tile(M, N, K) == tile
        if gated:
            _product(M, N, K, "swiglu")
            _product(M, N, K, "swiglu", seed=1, wide=3)
        else:
            for i, out in enumerate(("bf16", "f32", "add")):
                _product(M, N, K, out, seed=i, wide=i + 3)


@pytest.mark.parametrize("M,N,K", [(1, 12288, 4096), (333, 4096, 2048), (2048, 2048, 512), (3000, 5000, 128), (700, 9000, 256), (1500, 2500, 384), (5, 100, 131056)])
def test_gemm_i8_large(M, N, K):
    _product(M, N, K, "bf16")
    _product(M, N, K, "add", seed=1, wide=4)


@pytest.mark.parametrize("M", [1, 16, 17, 100, 700])
@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gemm_i8_residuals(M, swiglu, dt):
    """A residual behind the gate, and one of its own memory for either output."""
    rng = _rng(8, M)
    N, K = 320, 528
    cols = N // 2 if swiglu else N
    x, w = rng.integers(-128, 128, (M, K), dtype=np.int8), rng.integers(-128, 128, (N, K), dtype=np.int8)
    sx, sw = rng.uniform(0.5, 2, M).astype(np.float32), (rng.uniform(0.5, 2, N) / (5000 * np.sqrt(K))).astype(np.float32)
    for wide in (0, 3):
        r, _ = _strided((M, cols), torch.float32, wide, 1.0)
        r.copy_(_cuda(rng.standard_normal((M, cols)).astype(np.float32)))
        o, whole = _strided((M, cols), dt, wide, 3.0)
        vb.vla_op_gemm_i8(_cuda(x), _cuda(sx), _pack(w, sw), r, o, N, swiglu)
        y, res = _ref_gemm(x, sx, w, sw, swiglu), r.cpu().numpy().astype(np.float64)
        own = np.abs(y) * (2.0 ** -17 if swiglu else 4 * U32) + 1e-37
        tol = own + np.abs(y + res) * (U32 if dt == torch.float32 else UB + U32)
        assert np.all(np.abs(o.double().cpu().numpy() - (y + res)) <= tol * (1 + 2.0 ** -8))
        assert bool((whole[:, cols:] == 3.0).all())


def test_nothing_to_do():
    """Tensors without rows, tokens or sequences."""
    e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    Wp = torch.zeros(vb.vla_op_w8_packed_bytes(64, 64), dtype=torch.uint8, device="cuda")
    vb.vla_op_norm_i8(e(0, 64), None, None, None, 0.0, e(0, 64, dtype=torch.int8), e(0, dtype=torch.float32))
    vb.vla_op_gemm_i8(e(0, 64, dtype=torch.int8), e(0, dtype=torch.float32), Wp, None, e(0, 64), 64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    vb.vla_op_attention_packed(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), i32(0, 0), e(0, 4, 64))
    o = torch.full((5, 4, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    vb.vla_op_attention_packed(o, o[:, :2], o[:, 2:], i32(0), o.clone())
    cache = torch.zeros(vb.vla_op_kv8_bytes(2, 2, 32, 64), dtype=torch.uint8, device="cuda")
    vb.vla_op_kv8_store(e(2, 0, 2, 64), e(2, 0, 2, 64), i32(0, 0), None, cache, 32)
    vb.vla_op_kv8_load(cache, 32, i32(0, 0), None, e(2, 0, 2, 64), e(2, 0, 2, 64))
    vb.vla_op_attention_kv8(e(2, 0, 4, 64), cache, 32, 2, i32(1, 1), e(2, 0, 4, 64), 32)
    assert not bool(cache.any())


def test_gemm_i8_extremes():
    """The largest sum of all: -128 * -128 over the deepest K."""
    K, N = 131056, 32
    for M in (1, 20):
        x, w = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
        o = torch.empty((M, N), device="cuda")
        vb.vla_op_gemm_i8(_cuda(x), torch.ones(M, device="cuda"), _pack(w, np.ones(N, np.float32)), None, o, N)
        assert bool((o == 16384.0 * K).all())


def test_gemm_i8_rows_keep_to_themselves():
    """A scale that is not finite reaches its own row only; a row's bits do not depend on the others of the call."""
    rng = _rng(5)
    N, K = 512, 1024
    w, sw = rng.integers(-127, 128, (N, K), dtype=np.int8), rng.uniform(1e-4, 1e-3, N).astype(np.float32)
    Wp = _pack(w, sw)
    x = _cuda(rng.integers(-127, 128, (600, K), dtype=np.int8))
    sx = _cuda(rng.uniform(0.5, 2, 600).astype(np.float32))
    base = torch.empty((600, N), device="cuda")
    vb.vla_op_gemm_i8(x, sx, Wp, None, base, N)
    for M in (1, 16, 40, 200):
        o = torch.empty((M, N), device="cuda")
        vb.vla_op_gemm_i8(x[:M], sx[:M], Wp, None, o, N)
        assert torch.equal(o, base[:M])
        bad = sx[:M].clone()
        bad[M // 2] = float("nan")
        vb.vla_op_gemm_i8(x[:M], bad, Wp, None, o, N)
        keep = torch.arange(M, device="cuda") != M // 2
        assert torch.equal(o[keep], base[:M][keep]) and bool(o[M // 2].isnan().all())


def test_norm_into_gemm_in_a_graph():
    """Norm with the residual's addition, gated product, rows into codes, product into the residual: eagerly, and
    captured and replayed with other inputs in the same memory."""
    rng = _rng(6)
    M, d, F = 37, 896, 4864
    h0 = [_cuda(rng.standard_normal((M, d)).astype(np.float32)) for _ in range(3)]
    add = _cuda(rng.standard_normal((M, d))).bfloat16()
    g = _cuda(rng.uniform(0.5, 1.5, d).astype(np.float32))
    Wgu = _pack(rng.integers(-127, 128, (2 * F, d), dtype=np.int8), rng.uniform(1e-4, 6e-4, 2 * F).astype(np.float32))
    Wd = _pack(rng.integers(-127, 128, (d, F), dtype=np.int8), rng.uniform(1e-4, 6e-4, d).astype(np.float32))
    h, c1, s1 = torch.empty((M, d), device="cuda"), torch.empty((M, d), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    y, c2, s2 = torch.empty((M, F), dtype=torch.bfloat16, device="cuda"), torch.empty((M, F), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")

    def step():
        vb.vla_op_norm_i8(h, add, h, g, 1e-6, c1, s1)
        vb.vla_op_gemm_i8(c1, s1, Wgu, None, y, 2 * F, True)
        vb.vla_op_norm_i8(y, None, None, None, 0.0, c2, s2)
        vb.vla_op_gemm_i8(c2, s2, Wd, h, h, d)
    want = []
    for x in h0:
        h.copy_(x)
        step()
        want.append(h.clone())
    assert all(bool(w.isfinite().all()) for w in want) and not torch.equal(want[0], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, w in zip(h0 * 2, want * 2):
        h.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, w)
