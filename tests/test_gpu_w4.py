"""Products with 4-bit weights against float64."""
import numpy as np
import pytest

import synth
import w4kv4_ref as ref

pytestmark = pytest.mark.gpu


def _weights(tag, N, K, group, zeros, exact):
    rng = np.random.default_rng(synth.seed_of("w4", *tag))
    G = -(-K // group)
    codes = rng.integers(0, 16, (N, K), dtype=np.uint8)
    s = 2.0 ** -rng.integers(1, 4, (N, G)) if exact else ref.bf16(rng.uniform(0.002, 0.01, (N, G)))
    z = None
    if zeros:
        z = rng.integers(0, 16, (N, G)).astype(np.float64) if exact else ref.bf16(rng.uniform(0, 15, (N, G)))
    return codes, s, z


def _packed(codes, s, z, group):
    import torch
    from paper_2608_14586_amd import binding as vb
    N, K = codes.shape
    Wp = torch.empty(vb.vla_op_w4_packed_bytes(N, K, group), dtype=torch.uint8, device="cuda")
    vb.vla_op_w4_pack(torch.from_numpy(codes).cuda(), ref.to_dev(s), None if z is None else ref.to_dev(z), Wp, group)
    return Wp


SIZES = [(1, 1, 8, 32), (1, 16, 128, 128), (2, 17, 136, 64), (3, 31, 24, 128), (4, 896, 896, 64), (5, 33, 1000, 32),
         (7, 100, 264, 128), (8, 257, 512, 64), (9, 40, 4096, 128), (13, 50, 1032, 32), (16, 64, 2048, 64),
         (17, 48, 256, 64), (40, 130, 520, 32)]


@pytest.mark.parametrize("M,N,K,group", SIZES)
@pytest.mark.parametrize("zeros", [False, True])
def test_gemv_w4_exact(M, N, K, group, zeros):
    """Whole numbers: every partial sum is a multiple of 1/8 below 2^21 (4096
    inputs of at most 3 times (16 + 15) + (16 + 15)), so fp32 holds each and the
    result is equal to the last bit, whatever the order."""
    import torch
    from paper_2608_14586_amd import binding as vb
    codes, s, z = _weights((M, N, K, group, zeros), N, K, group, zeros, True)
    x = np.random.default_rng(synth.seed_of("w4x", M, K)).integers(-3, 4, (M, K)).astype(np.float64)
    y = torch.full((M, N), 7.0, dtype=torch.float32, device="cuda")
    vb.vla_op_gemv_w4(ref.to_dev(x), _packed(codes, s, z, group), None, y, N, group)
    assert np.array_equal(ref.from_dev(y), x @ ref.w4_weights(codes, s, z, group).T)


def _bound(x, codes, s, z, group):
    """Accumulation error of the product: in a group each MFMA step rounds the
    running sums of (16 + c) x and of x, both at most 31 sum |x| after the
    factor 16 + z, and three more roundings join them; then one rounding a
    group and wave of the total.  Factor 4."""
    N, K = codes.shape
    k = np.arange(K) // group
    ax = np.abs(x) @ s[:, k].T
    mag = np.abs(x) @ np.abs(ref.w4_weights(codes, s, z, group)).T
    return 4 * 2.0 ** -24 * (62 * (group / 32 + 3) * ax + (-(-K // group) + 10) * mag), mag


@pytest.mark.parametrize("M,N,K,group,zeros", [(1, 200, 4096, 128, False), (4, 96, 11008, 32, True),
                                               (13, 64, 1544, 64, True), (6, 61, 200, 128, True)])
@pytest.mark.parametrize("out", ["f32", "bf16", "add"])
def test_gemv_w4(M, N, K, group, zeros, out):
    import torch
    from paper_2608_14586_amd import binding as vb
    codes, s, z = _weights((M, N, K, group), N, K, group, zeros, False)
    x = ref.normal(("w4x", M, K), (M, K))
    want = x @ ref.w4_weights(codes, s, z, group).T
    bound, _ = _bound(x, codes, s, z, group)
    Wp = _packed(codes, s, z, group)
    y = torch.empty((M, N), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
    res = None
    if out == "add":  # in place
        h = synth.normal_f32(synth.seed_of("w4h", M, N), (M, N))
        y.copy_(torch.from_numpy(h))
        want, bound, res = want + h, bound + 2.0 ** -23 * (np.abs(want) + np.abs(h)), y
    vb.vla_op_gemv_w4(ref.to_dev(x), Wp, res, y, N, group)
    if out == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    assert (np.abs(ref.from_dev(y) - want) <= bound).all()


@pytest.mark.parametrize("M,F,K,group,f32", [(1, 16, 64, 32, True), (4, 688, 256, 64, False), (9, 48, 1032, 128, True),
                                             (16, 1376, 512, 128, False)])
def test_gemv_w4_swiglu(M, F, K, group, f32):
    """silu(gate) up: the product's error through silu's slope (at most 1.1)
    and the other factor, the exponential and division (2^-20 relative), and
    the rounding of a bf16 result."""
    import torch
    from paper_2608_14586_amd import binding as vb
    codes, s, z = _weights((M, F, K, group), 2 * F, K, group, True, False)
    x = ref.normal(("w4x", M, K), (M, K))
    y = x @ ref.w4_weights(codes, s, z, group).T
    b, _ = _bound(x, codes, s, z, group)
    g, u = y[:, :F], y[:, F:]
    sg = g / (1 + np.exp(-g))
    want = sg * u
    out = torch.empty((M, F), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    vb.vla_op_gemv_w4(ref.to_dev(x), _packed(codes, s, z, group), None, out, 2 * F, group, True)
    bound = 1.1 * b[:, :F] * (np.abs(u) + b[:, F:]) + np.abs(sg) * b[:, F:] + 2.0 ** -20 * np.abs(want)
    if not f32:
        bound += 2.0 ** -8 * np.abs(want)
    assert (np.abs(ref.from_dev(out) - want) <= bound + 1e-30).all()


def test_gemv_w4_swiglu_and_residual():
    """The gated product on top of a residual, in place in fp32."""
    import torch
    from paper_2608_14586_amd import binding as vb
    M, F, K, group = 5, 80, 192, 64
    codes, s, z = _weights((M, F, K, group), 2 * F, K, group, True, False)
    x = ref.normal(("w4x", M, K), (M, K))
    y = x @ ref.w4_weights(codes, s, z, group).T
    b, _ = _bound(x, codes, s, z, group)
    g, u = y[:, :F], y[:, F:]
    h0 = synth.normal_f32(synth.seed_of("w4sh", M, F), (M, F))
    h = torch.from_numpy(h0.copy()).cuda()
    vb.vla_op_gemv_w4(ref.to_dev(x), _packed(codes, s, z, group), h, h, 2 * F, group, True)
    sg = g / (1 + np.exp(-g))
    want = h0 + sg * u
    bound = 1.1 * b[:, :F] * (np.abs(u) + b[:, F:]) + np.abs(sg) * b[:, F:] + 2.0 ** -20 * np.abs(sg * u) + 2.0 ** -23 * (np.abs(want) + np.abs(h0))
    assert (np.abs(ref.from_dev(h) - want) <= bound).all()


def test_gemv_w4_strides_and_neighbours():
    """Rows of x inside a wider array, rows of out with a tail that stays as it
    was, and a row of x that is not finite: it reaches no other row."""
    import torch
    from paper_2608_14586_amd import binding as vb
    M, N, K, group = 11, 37, 200, 64
    codes, s, z = _weights((M, N, K), N, K, group, True, True)
    x = np.random.default_rng(3).integers(-3, 4, (M, K)).astype(np.float64)
    wide = torch.full((M, K + 56), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 16:16 + K] = ref.to_dev(x)
    wide[4, 16 + 77] = float("inf")
    y = torch.full((M + 2, N + 5), 9.0, dtype=torch.float32, device="cuda")
    vb.vla_op_gemv_w4(wide[:, 16:16 + K], _packed(codes, s, z, group), None, y[:M, :N], N, group)
    got, want = ref.from_dev(y), x @ ref.w4_weights(codes, s, z, group).T
    rows = [m for m in range(M) if m != 4]
    assert np.array_equal(got[:M, :N][rows], want[rows])
    assert not np.isfinite(got[4, :N]).any()
    assert (got[M:] == 9).all() and (got[:, N:] == 9).all()


def test_gemv_w4_on_a_stream_and_in_a_graph():
    import torch
    from paper_2608_14586_amd import binding as vb
    M, N, K, group = 3, 96, 640, 128
    codes, s, z = _weights((M, N, K), N, K, group, True, True)
    Wp = _packed(codes, s, z, group)
    w = ref.w4_weights(codes, s, z, group)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((M, N), dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        vb.vla_op_gemv_w4(x, Wp, None, y, N, group, stream=torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        v = np.random.default_rng(i).integers(-3, 4, (M, K)).astype(np.float64)
        x.copy_(ref.to_dev(v))
        y.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ref.from_dev(y), v @ w.T), i
    with torch.cuda.stream(side):
        x.copy_(ref.to_dev(-v))
        vb.vla_op_gemv_w4(x, Wp, None, y, N, group, stream=side.cuda_stream)
    side.synchronize()
    assert np.array_equal(ref.from_dev(y), -v @ w.T)


@pytest.mark.parametrize("M,N,K,group,swiglu", [
    (3, 4096, 2568, 64, False), (13, 4112, 2568, 32, False), (1, 4096, 4104, 32, False), (12, 4112, 4104, 64, False),
    (5, 4112, 1032, 128, False), (6, 8224, 1024, 64, True), (20, 2048, 2696, 128, False), (5, 8192, 136, 64, False),
    (16, 8208, 264, 128, False), (2, 8208, 264, 32, False), (1, 8192, 2568, 32, True), (7, 8224, 2568, 128, True),
    (9, 16416, 136, 64, True),
    (1, 20520, 136, 32, False), (3, 12330, 1544, 64, False), (2, 4130, 3336, 128, False), (6, 12330, 136, 128, False),
    (7, 4130, 520, 32, False), (5, 4130, 8200, 64, False), (8, 41000, 136, 64, False), (6, 12340, 2568, 128, False),
    (13, 41000, 136, 32, False), (16, 12340, 2568, 64, False), (30, 12330, 136, 128, False), (1, 152070, 264, 64, False),
    (6, 41056, 136, 32, True), (8, 8224, 2568, 64, True), (11, 41056, 136, 128, True), (16, 8224, 2568, 32, True),
    (2, 152096, 136, 32, True)])
def test_gemv_w4_either_side_of_a_choice(M, N, K, group, swiglu):
    """Sizes that take each number of waves and tiles, with ends inside a
    workgroup's tiles."""
    import torch
    from paper_2608_14586_amd import binding as vb
    codes, s, z = _weights((M, N, K, group), N, K, group, True, True)
    x = np.random.default_rng(M + N).integers(-3, 4, (M, K)).astype(np.float64)
    want = x @ ref.w4_weights(codes, s, z, group).T
    bound = np.zeros(want.shape)
    if swiglu:
        # e^-v is 2^(-v log2 e): the constant's rounding and the product's are at
        # most 2^-24 of the exponent each, so e^-v is off by |v| 2^-23 of itself; the
        # instruction, a sum, a division and a product add less than 2^-20.  Below
        # v = -88 e^-v overflows and the result is 0 for less than 2^-100.
        v = want[:, :N // 2]
        want = v / (1 + np.exp(np.minimum(-v, 700))) * want[:, N // 2:]
        bound = (2.0 ** -20 + 2.0 ** -23 * np.abs(v)) * np.abs(want) + 2.0 ** -100
    y = torch.full(want.shape, 7.0, dtype=torch.float32, device="cuda")
    vb.vla_op_gemv_w4(ref.to_dev(x), _packed(codes, s, z, group), None, y, N, group, swiglu)
    assert (np.abs(ref.from_dev(y) - want) <= bound).all()
