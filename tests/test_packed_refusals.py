"""What attention over packed prompts refuses, on the CPU: no pointer is read."""
import struct

import pytest

from paper_2608_14586_amd import binding as vb

P = 1 << 20  # an address that is never read


def _h(p=P, seq=0, token=8, head=8):
    return struct.pack("Pqqq", p or 0, seq, token, head)


ARGS = dict(q=_h(), k=_h(), v=_h(), offsets=P, o=_h(), n_seq=2, T=10, H=4, Hkv=2, dh=64, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), "INVALID_ARG"), (dict(k=_h(None)), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(o=_h(None)), "INVALID_ARG"),
    (dict(offsets=None), "INVALID_ARG"), (dict(n_seq=-1), "INVALID_ARG"), (dict(T=-1), "INVALID_ARG"), (dict(H=0), "INVALID_ARG"),
    (dict(Hkv=-2), "INVALID_ARG"), (dict(k=_h(token=-8)), "INVALID_ARG"), (dict(o=_h(token=0)), "INVALID_ARG"), (dict(o=_h(head=0)), "INVALID_ARG"),
    (dict(Hkv=3), "UNSUPPORTED"), (dict(dh=96), "UNSUPPORTED"), (dict(q=_h(P + 8)), "UNSUPPORTED"), (dict(v=_h(head=4)), "UNSUPPORTED"),
    (dict(o=_h(token=12)), "UNSUPPORTED"), (dict(offsets=P + 2), "UNSUPPORTED"), (dict(k=_h(token=1 << 24)), "UNSUPPORTED"),
    (dict(v=_h(token=1 << 40)), "UNSUPPORTED"), (dict(T=2147483647, H=128, Hkv=128), "UNSUPPORTED"), (dict(n_seq=1 << 30), "UNSUPPORTED")])
def test_refuses(change, code):
    assert vb.STATUS[vb.lib().vla_op_attention_packed(*{**ARGS, **change}.values())] == "VLA_ERR_" + code


def test_nothing_to_do():
    z = _h(None)
    assert vb.lib().vla_op_attention_packed(z, z, z, P, z, 2, 0, 4, 2, 64, None) == 0
    assert vb.lib().vla_op_attention_packed(_h(), _h(), _h(), None, _h(), 0, 10, 4, 2, 64, None) == 0


def test_binding_refuses_before_the_library():
    import torch
    q, k = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        vb.vla_op_attention_packed(q, k, k, torch.zeros(2, dtype=torch.int32), q)
