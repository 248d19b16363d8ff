"""The largest row stride of x that products with 4-bit weights take, on the CPU."""
import pytest

from paper_2608_14586_amd import binding as vb

P = 1 << 20  # an address that is never read


@pytest.mark.parametrize("ldx", [((1 << 30) - 256) // 15 // 8 * 8 + 8, 1 << 31, 1 << 60, (1 << 63) - 8] +
                         [(j << 63) // 15 // 8 * 8 + 8 for j in range(1, 15)])
@pytest.mark.parametrize("M", [2, 16, 17])
def test_rows_past_two_gigabytes_are_refused(ldx, M):
    """Also where 15 strides, or the bytes in them, pass 64 bits and come out small."""
    code = vb.lib().vla_op_gemv_w4(P, ldx, P, None, P, 64, vb.VLA_F32, 0, M, 64, 256, 64, None)
    assert vb.STATUS[code] == "VLA_ERR_UNSUPPORTED"
