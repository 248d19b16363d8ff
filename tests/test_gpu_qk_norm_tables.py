"""Rotary tables without a row."""
import pytest

import w4kv4_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_no_position_has_a_row(norm, given):
    """Every token is padding: its rows of q_out and k_out stay as they were."""
    import torch
    from paper_2608_14586_amd import binding as vb
    B, L, H, Hkv, dh = 2, 3, 4, 2, 64
    q, k = ref.to_dev(ref.normal(("tq",), (B, L, H, dh))), ref.to_dev(ref.normal(("tk",), (B, L, Hkv, dh)))
    table = torch.empty((0, dh // 2), device="cuda")
    g = torch.ones(dh, device="cuda") if norm else None
    pos = torch.zeros((B, L), dtype=torch.int32, device="cuda") if given else None
    q_out, k_out = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    vb.vla_op_qk_norm_rope(q, k, g, g, 1e-6, table, table, pos, q_out, k_out)
    assert (q_out == 3).all() and (k_out == 3).all()
    for cos, sin in ((table, None), (None, table)):
        with pytest.raises(vb.VlaError) as e:
            vb.vla_op_qk_norm_rope(q, k, g, g, 1e-6, cos, sin, pos, q_out, k_out)
        assert e.value.name == "VLA_ERR_INVALID_ARG"
