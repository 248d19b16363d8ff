"""What the 8-bit row and product operators refuse, and their sizes, on the CPU: every
call here returns before any GPU work (no pointer is read)."""
import pytest

from paper_2608_14586_amd import binding as vb

P = 1 << 20  # an address that is never read


def _name(code):
    return vb.STATUS[code]


NORM = dict(x=P, ldx=64, xt=vb.VLA_F32, add=P, ldadd=64, at=vb.VLA_BF16, sum=P, ldsum=64, g=P, eps=1e-6, codes=P, ldc=64,
            scales=P, M=2, d=64, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), "INVALID_ARG"), (dict(codes=None), "INVALID_ARG"), (dict(scales=None), "INVALID_ARG"),
    (dict(M=-1), "INVALID_ARG"), (dict(d=0), "INVALID_ARG"), (dict(xt=7), "INVALID_ARG"), (dict(at=3), "INVALID_ARG"),
    (dict(eps=-1.0), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"), (dict(ldx=56), "INVALID_ARG"),
    (dict(ldadd=-8), "INVALID_ARG"), (dict(ldadd=0), "INVALID_ARG"), (dict(ldsum=8), "INVALID_ARG"), (dict(ldc=0), "INVALID_ARG"),
    (dict(d=60), "UNSUPPORTED"), (dict(d=32776, ldx=1 << 16, ldadd=1 << 16, ldsum=1 << 16, ldc=1 << 16), "UNSUPPORTED"),
    (dict(ldx=68), "UNSUPPORTED"), (dict(ldc=68), "UNSUPPORTED"), (dict(ldsum=65), "UNSUPPORTED"), (dict(x=P + 8), "UNSUPPORTED"),
    (dict(add=P + 2), "UNSUPPORTED"), (dict(sum=P + 4), "UNSUPPORTED"), (dict(g=P + 4), "UNSUPPORTED"),
    (dict(codes=P + 4), "UNSUPPORTED"), (dict(scales=P + 2), "UNSUPPORTED"), (dict(M=1 << 22), "UNSUPPORTED")])
def test_norm_i8_refuses(change, code):
    assert _name(vb.lib().vla_op_norm_i8(*{**NORM, **change}.values())) == "VLA_ERR_" + code


@pytest.mark.parametrize("args,code", [
    ((None, P, P, 16, 64, None), "INVALID_ARG"), ((P, None, P, 16, 64, None), "INVALID_ARG"), ((P, P, None, 16, 64, None), "INVALID_ARG"),
    ((P, P, P, 0, 64, None), "INVALID_ARG"), ((P, P, P, 16, -16, None), "INVALID_ARG"), ((P, P, P, 16, 72, None), "UNSUPPORTED"),
    ((P, P, P, 16, 131072, None), "UNSUPPORTED"), ((P, P, P, 1 << 25, 64, None), "UNSUPPORTED"), ((P + 8, P, P, 16, 64, None), "UNSUPPORTED"),
    ((P, P + 2, P, 16, 64, None), "UNSUPPORTED"), ((P, P, P + 8, 16, 64, None), "UNSUPPORTED")])
def test_w8_pack_refuses(args, code):
    assert _name(vb.lib().vla_op_w8_pack(*args)) == "VLA_ERR_" + code


GEMM = dict(x=P, ldx=256, sx=P, Wp=P, residual=None, out=P, ldo=64, out_dtype=vb.VLA_F32, swiglu=0, M=2, N=64, K=256, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), "INVALID_ARG"), (dict(sx=None), "INVALID_ARG"), (dict(Wp=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(M=-1), "INVALID_ARG"), (dict(N=0), "INVALID_ARG"), (dict(K=-16), "INVALID_ARG"), (dict(out_dtype=2), "INVALID_ARG"),
    (dict(ldx=-16), "INVALID_ARG"), (dict(ldx=240), "INVALID_ARG"), (dict(ldo=63), "INVALID_ARG"),
    (dict(K=250), "UNSUPPORTED"), (dict(K=1 << 17, ldx=1 << 17), "UNSUPPORTED"), (dict(ldx=264), "UNSUPPORTED"), (dict(x=P + 8), "UNSUPPORTED"),
    (dict(Wp=P + 4), "UNSUPPORTED"), (dict(sx=P + 1), "UNSUPPORTED"), (dict(out=P + 2), "UNSUPPORTED"), (dict(residual=P + 1), "UNSUPPORTED"),
    (dict(swiglu=1, N=96), "UNSUPPORTED"), (dict(ldx=1 << 23), "UNSUPPORTED"), (dict(ldo=1 << 21), "UNSUPPORTED"),
    (dict(N=1 << 25, ldo=1 << 25), "UNSUPPORTED"), (dict(M=2147483647, N=(1 << 25) - 32, ldo=1 << 25), "UNSUPPORTED")])
def test_gemm_i8_refuses(change, code):
    assert _name(vb.lib().vla_op_gemm_i8(*{**GEMM, **change}.values())) == "VLA_ERR_" + code


def test_nothing_to_do():
    L = vb.lib()
    assert L.vla_op_gemm_i8(*{**GEMM, "M": 0, "x": None, "sx": None, "out": None}.values()) == 0
    assert L.vla_op_norm_i8(*{**NORM, "M": 0, "x": None, "codes": None, "scales": None}.values()) == 0


def test_sizes():
    assert vb.vla_op_w8_packed_bytes(32, 256) == 32 * 256 + 32 * 4
    assert vb.vla_op_w8_packed_bytes(33, 272) == 64 * 512 + 64 * 4  # whole pairs of tiles, whole runs of four steps
    assert vb.vla_op_w8_packed_bytes(1 << 20, 1 << 14) == (1 << 34) + (1 << 22)  # past 32 bits
    for bad in ((0, 64), (16, 0), (16, 24), (-1, 64), (16, 131072), (1 << 25, 64)):
        assert vb.vla_op_w8_packed_bytes(*bad) == 0


def test_binding_refuses_before_the_library():
    """Tensors that do not fit raise ValueError (host tensors among them)."""
    import torch
    x, s = torch.zeros((2, 256), dtype=torch.int8), torch.zeros(2)
    y = torch.zeros((2, 64))
    Wp = torch.zeros(vb.vla_op_w8_packed_bytes(64, 256), dtype=torch.uint8)
    for call in (lambda: vb.vla_op_gemm_i8(x, s, Wp, None, y, 64), lambda: vb.vla_op_norm_i8(y, None, None, None, 0.0, x, s),
                 lambda: vb.vla_op_w8_pack(x, s, Wp), lambda: vb.vla_op_w8_pack(None, s, Wp)):
        with pytest.raises(ValueError):
            call()



def test_tiles():
    """The shapes that the GPU tests run in every tile do take it."""
    from i8_tiles import TILES
    assert len(TILES) == 10
    for tile, shapes in TILES.items():
        for M, N, K, gated in shapes:
            assert vb.vla_op_gemm_i8_tile(M, N, K) == tile and (not gated or N % 64 == 0)
    for bad in ((0, 64, 64), (-1, 64, 64), (20, 0, 64), (20, 64, 24)):
        with pytest.raises(vb.VlaError):
            vb.vla_op_gemm_i8_tile(*bad)
