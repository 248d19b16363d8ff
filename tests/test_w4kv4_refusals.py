"""What the 4-bit operators refuse, and their sizes, on the CPU: every call here
returns before any GPU work (no pointer is read)."""
import struct

import pytest

from paper_2608_14586_amd import binding as vb

P = 1 << 20  # an address that is never read


def _h(p=P, seq=8, token=8, head=8):
    return struct.pack("Pqqq", p or 0, seq, token, head)


def _name(code):
    return vb.STATUS[code]


GEMV = dict(x=P, ldx=256, Wp=P, residual=None, out=P, ldo=64, out_dtype=vb.VLA_F32, swiglu=0, M=2, N=64, K=256, group=64,
            stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), "INVALID_ARG"), (dict(Wp=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(M=-1), "INVALID_ARG"), (dict(N=0), "INVALID_ARG"), (dict(K=-8), "INVALID_ARG"), (dict(out_dtype=2), "INVALID_ARG"),
    (dict(ldx=-8), "INVALID_ARG"), (dict(ldx=248), "INVALID_ARG"), (dict(ldo=63), "INVALID_ARG"),
    (dict(K=252, ldx=256), "UNSUPPORTED"), (dict(group=16), "UNSUPPORTED"), (dict(group=0), "UNSUPPORTED"),
    (dict(group=256), "UNSUPPORTED"), (dict(ldx=260), "UNSUPPORTED"), (dict(x=P + 8), "UNSUPPORTED"),
    (dict(Wp=P + 4), "UNSUPPORTED"), (dict(out=P + 2), "UNSUPPORTED"), (dict(residual=P + 1), "UNSUPPORTED"),
    (dict(swiglu=1, N=48), "UNSUPPORTED"), (dict(N=(1 << 25) + 1, ldo=1 << 26), "UNSUPPORTED"), (dict(ldx=1 << 30), "UNSUPPORTED"), (dict(M=16 * 65535 + 1), "UNSUPPORTED")])
def test_gemv_w4_refuses(change, code):
    assert _name(vb.lib().vla_op_gemv_w4(*{**GEMV, **change}.values())) == "VLA_ERR_" + code


def test_nothing_to_do():
    """No rows, no sequences or no tokens: fine, and nothing is launched."""
    L = vb.lib()
    assert L.vla_op_gemv_w4(*{**GEMV, "M": 0, "x": None, "out": None}.values()) == 0
    z = _h(None)
    for B, n in ((0, 4), (3, 0)):
        assert L.vla_op_qk_norm_rope(z, z, vb.VLA_BF16, None, None, 0.0, None, None, 0, None, z, z, B, n, 2, 1, 64, None) == 0
        assert L.vla_op_kv4_store(z, z, None, None, P, B, n, 2, 32, 64, None) == 0
        assert L.vla_op_kv4_load(P, None, None, z, z, B, n, 2, 32, 64, None) == 0
        assert L.vla_op_attention_kv4(z, P, P, z, B, n, 2, 2, 32, 64, 32, 0, 0, None, 0, None) == 0


def test_sizes():
    assert vb.vla_op_w4_packed_bytes(16, 128, 128) == 16 * 128 // 2 + 16 * 4
    assert vb.vla_op_w4_packed_bytes(17, 136, 32) == 2 * 2 * (1024 + 16 * 4 * 4)
    assert vb.vla_op_w4_packed_bytes(1 << 17, 1 << 14, 64) == (1 << 31) // 2 + (1 << 31) // 16
    for bad in ((0, 128, 128), (16, 0, 128), (16, 132, 128), (16, 128, 48), (-1, 128, 32)):
        assert vb.vla_op_w4_packed_bytes(*bad) == 0
    assert vb.vla_op_kv4_bytes(2, 3, 64, 128) == 2 * 3 * 64 * 2 * (64 + 16)
    assert vb.vla_op_kv4_bytes(64, 8, 1 << 20, 128) == 64 * 8 * (1 << 20) * 160  # past 32 bits
    for bad in ((-1, 1, 32, 64), (1, 0, 32, 64), (1, 1, 33, 64), (1, 1, 0, 64), (1, 1, 32, 96), (1, 1, 1 << 25, 64)):
        assert vb.vla_op_kv4_bytes(*bad) == 0
    assert vb.vla_op_attention_kv4_scratch(1, 1, 32, 32, 128, 32) == 0  # one split
    long = vb.vla_op_attention_kv4_scratch(1, 1, 32, 8, 128, 1 << 20)
    assert long > 0
    assert vb.vla_op_attention_kv4_scratch(1, 1, 32, 8, 128, 1 << 20, 1 << 20, 4) == long  # a window that hides nothing
    assert vb.vla_op_attention_kv4_scratch(1, 1, 32, 8, 128, 1 << 20, 1 << 30, 4) == long
    assert vb.vla_op_attention_kv4_scratch(1, 1, 32, 5, 128, 4096) == 0


@pytest.mark.parametrize("args,code", [
    ((None, P, None, P, 16, 128, 32, None), "INVALID_ARG"), ((P, None, None, P, 16, 128, 32, None), "INVALID_ARG"),
    ((P, P, None, None, 16, 128, 32, None), "INVALID_ARG"), ((P, P, None, P, 0, 128, 32, None), "INVALID_ARG"),
    ((P, P, None, P, 16, 100, 32, None), "UNSUPPORTED"), ((P, P, None, P, 16, 128, 24, None), "UNSUPPORTED"),
    ((P, P, None, P + 8, 16, 128, 32, None), "UNSUPPORTED"), ((P, P + 1, None, P, 16, 128, 32, None), "UNSUPPORTED"),
    ((P, P, P + 1, P, 16, 128, 32, None), "UNSUPPORTED")])
def test_pack_refuses(args, code):
    assert _name(vb.lib().vla_op_w4_pack(*args)) == "VLA_ERR_" + code


QK = dict(q=_h(), k=_h(), dt=vb.VLA_BF16, gq=P, gk=P, eps=1e-6, cos=P, sin=P, n_pos=4, pos=P, qo=_h(), ko=_h(), B=2, L=3, H=4,
          Hkv=2, dh=64, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), "INVALID_ARG"), (dict(ko=None), "INVALID_ARG"), (dict(q=_h(None)), "INVALID_ARG"),
    (dict(cos=None), "INVALID_ARG"), (dict(sin=None), "INVALID_ARG"), (dict(n_pos=-1), "INVALID_ARG"),
    (dict(B=-1), "INVALID_ARG"), (dict(H=0), "INVALID_ARG"), (dict(Hkv=0), "INVALID_ARG"), (dict(dt=5), "INVALID_ARG"),
    (dict(eps=-1e-6), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"),
    (dict(q=_h(seq=-8)), "INVALID_ARG"), (dict(qo=_h(token=0)), "INVALID_ARG"), (dict(ko=_h(head=0)), "INVALID_ARG"),
    (dict(dh=96), "UNSUPPORTED"), (dict(q=_h(P + 2)), "UNSUPPORTED"), (dict(ko=_h(head=4)), "UNSUPPORTED"),
    (dict(gq=P + 4), "UNSUPPORTED"), (dict(sin=P + 8), "UNSUPPORTED"), (dict(pos=P + 2), "UNSUPPORTED"),
    (dict(B=1 << 20, L=1 << 20), "UNSUPPORTED")])
def test_qk_norm_rope_refuses(change, code):
    assert _name(vb.lib().vla_op_qk_norm_rope(*{**QK, **change}.values())) == "VLA_ERR_" + code


KV = dict(k=_h(), v=_h(), start=P, count=P, cache=P, B=2, L=3, Hkv=2, L_cap=64, dh=64, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(k=None), "INVALID_ARG"), (dict(v=_h(None)), "INVALID_ARG"), (dict(cache=None), "INVALID_ARG"),
    (dict(B=-1), "INVALID_ARG"), (dict(L=-1), "INVALID_ARG"), (dict(Hkv=0), "INVALID_ARG"), (dict(L_cap=0), "INVALID_ARG"),
    (dict(v=_h(head=-8)), "INVALID_ARG"), (dict(L_cap=65), "UNSUPPORTED"), (dict(L_cap=1 << 25), "UNSUPPORTED"),
    (dict(dh=80), "UNSUPPORTED"), (dict(cache=P + 8), "UNSUPPORTED"), (dict(k=_h(token=12)), "UNSUPPORTED"),
    (dict(start=P + 1), "UNSUPPORTED"), (dict(B=1 << 14, L=1 << 30), "UNSUPPORTED")])
def test_kv4_rows_refuse(change, code):
    a = {**KV, **change}
    assert _name(vb.lib().vla_op_kv4_store(*a.values())) == "VLA_ERR_" + code
    order = ("cache", "start", "count", "k", "v", "B", "L", "Hkv", "L_cap", "dh", "stream")
    assert _name(vb.lib().vla_op_kv4_load(*(a[n] for n in order))) == "VLA_ERR_" + code


def test_kv4_load_refuses_rows_that_coincide():
    """Rows may be read many times (a stride of 0), not written."""
    for h in (_h(seq=0), _h(token=0), _h(head=0)):
        a = (P, None, None, h, _h(), 2, 3, 2, 64, 64, None)
        assert _name(vb.lib().vla_op_kv4_load(*a)) == "VLA_ERR_INVALID_ARG"


ATT = dict(q=_h(), cache=P, lens=P, o=_h(), B=1, Lq=1, H=4, Hkv=2, L_cap=4096, dh=64, max_len=4096, window=0, sinks=0,
           scratch=P, nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), "INVALID_ARG"), (dict(o=_h(None)), "INVALID_ARG"), (dict(cache=None), "INVALID_ARG"),
    (dict(lens=None), "INVALID_ARG"), (dict(B=-1), "INVALID_ARG"), (dict(Lq=-1), "INVALID_ARG"), (dict(H=0), "INVALID_ARG"),
    (dict(max_len=-1), "INVALID_ARG"), (dict(window=-1), "INVALID_ARG"), (dict(sinks=-1), "INVALID_ARG"),
    (dict(scratch=None), "INVALID_ARG"), (dict(o=_h(head=0)), "INVALID_ARG"), (dict(q=_h(head=-8)), "INVALID_ARG"),
    (dict(H=5), "UNSUPPORTED"), (dict(dh=256), "UNSUPPORTED"), (dict(L_cap=4097), "UNSUPPORTED"),
    (dict(q=_h(P + 4)), "UNSUPPORTED"), (dict(o=_h(seq=4)), "UNSUPPORTED"), (dict(scratch=P + 4), "UNSUPPORTED"),
    (dict(cache=P + 2), "UNSUPPORTED"), (dict(B=1 << 20, H=64, Hkv=32), "UNSUPPORTED"), (dict(Lq=1 << 30), "UNSUPPORTED"),
    (dict(Lq=1 << 19), "UNSUPPORTED"), (dict(max_len=4097), "SHAPE"), (dict(nbytes=4), "SHAPE"),
    (dict(scratch=None, nbytes=0), "SHAPE")])
def test_attention_kv4_refuses(change, code):
    assert _name(vb.lib().vla_op_attention_kv4(*{**ATT, **change}.values())) == "VLA_ERR_" + code


def test_binding_refuses_before_the_library():
    """Tensors that do not fit raise ValueError (host tensors among them)."""
    import torch
    x = torch.zeros((2, 256), dtype=torch.bfloat16)
    y = torch.zeros((2, 64))
    Wp = torch.zeros(vb.vla_op_w4_packed_bytes(64, 256, 64), dtype=torch.uint8)
    h = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    lens = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: vb.vla_op_gemv_w4(x, Wp, None, y, 64, 64), lambda: vb.vla_op_qk_norm_rope(h, h, None, None, 0.0, None, None, None, h, h),
                 lambda: vb.vla_op_kv4_store(h, h, None, None, Wp, 32), lambda: vb.vla_op_kv4_load(Wp, 32, None, None, h, h),
                 lambda: vb.vla_op_attention_kv4(h, Wp, 32, 2, lens, h, 32),
                 lambda: vb.vla_op_w4_pack(Wp.view(-1, 8), y, None, Wp, 32)):
        with pytest.raises(ValueError):
            call()
