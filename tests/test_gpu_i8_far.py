"""Rows and weights further apart than 32 bits reach: the bits of the same call on rows side by side."""
import numpy as np
import pytest
import torch

from paper_2608_14586_amd import binding as vb

pytestmark = pytest.mark.gpu


def _far(rows, stride, wide, dtype, fill=None):
    """[rows][wide] with rows that far apart, the memory between them untouched."""
    whole = torch.empty(rows * stride, dtype=dtype, device="cuda")
    x = whole.as_strided((rows, wide), (stride, 1))
    if fill is not None:
        x.copy_(fill)
    return x


def _rng(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(k * 1000 ** i for i, k in enumerate(key)))
    return g


def test_norm():
    M, d, far = 1100, 512, 1 << 21  # 2.3 10^9 elements
    g = _rng(1)
    x, y = (torch.randn((M, d), device="cuda", generator=g) for _ in range(2))
    gain = torch.rand(d, device="cuda", generator=g) + 0.5
    want = torch.empty((M, d), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    vb.vla_op_norm_i8(x, y, None, gain, 1e-6, *want)
    fx = _far(M, far, d, torch.float32, x)
    codes, scales = _far(M, far, d, torch.int8), torch.empty(M, device="cuda")
    vb.vla_op_norm_i8(fx, y, fx, gain, 1e-6, codes, scales)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1]) and torch.equal(fx, x + y)


@pytest.mark.parametrize("N", [64, 300])
def test_rows_of_a_product(N):
    M, K = 1100, 320
    g = _rng(2, N)
    x = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    sx = torch.rand(M, device="cuda", generator=g)
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    Wp = torch.empty(vb.vla_op_w8_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    vb.vla_op_w8_pack(w, torch.rand(N, device="cuda", generator=g), Wp)
    r = torch.randn((M, N), device="cuda", generator=g)
    want = torch.empty_like(r)
    vb.vla_op_gemm_i8(x, sx, Wp, r, want, N)
    out = _far(M, 1 << 20, N, torch.float32, r)                      # 4.6 10^9 bytes
    vb.vla_op_gemm_i8(_far(M, 1 << 22, K, torch.int8, x), sx, Wp, out, out, N)  # 4.6 10^9 bytes of x
    assert torch.equal(out, want)


@pytest.mark.parametrize("M", [1, 20, 200])
def test_weights_past_32_bits(M):
    """33024 rows of 131056 codes, 4.3 10^9 bytes; the last and some others in 64 bits."""
    N, K = 33024, 131056
    g = _rng(3)
    x = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    Wp = torch.empty(vb.vla_op_w8_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    vb.vla_op_w8_pack(w, torch.ones(N, device="cuda"), Wp)
    out = torch.empty((M, N), device="cuda")
    vb.vla_op_gemm_i8(x, torch.ones(M, device="cuda"), Wp, None, out, N)
    some = torch.cat([torch.arange(64), torch.randint(0, N, (64,)), torch.arange(N - 96, N)]).cuda()
    want = x.double() @ w[some].double().t().contiguous()  # whole numbers below 2^31, which 53 bits hold
    assert torch.equal(out[:, some], want.float())


@pytest.mark.parametrize("dh", [64, 128])
def test_packed_prompts(dh):
    T, H, Hkv, far = 700, 4, 2, (1 << 24) - 8  # 1.2 10^10 elements
    g = _rng(4, dh)
    q, k, v = (torch.randn((T, n, dh), device="cuda", generator=g).bfloat16() for n in (H, Hkv, Hkv))
    offsets = torch.tensor([0, 333, 334, 690], dtype=torch.int32, device="cuda")
    want = torch.zeros_like(q)
    vb.vla_op_attention_packed(q, k, v, offsets, want)
    whole = torch.empty(T * far, dtype=torch.bfloat16, device="cuda")
    at, views = 0, []
    for t in (q, k, v, want):
        views.append(whole.as_strided(t.shape, (far, dh, 1), at))
        at += t.shape[1] * dh
    for to, t in zip(views, (q, k, v, torch.zeros_like(q))):
        to.copy_(t)
    vb.vla_op_attention_packed(*views[:3], offsets, views[3])
    assert torch.equal(views[3], want) and bool(torch.isfinite(want).all())
    assert np.count_nonzero(want[690:].float().cpu().numpy()) == 0
