"""The Swish constants that a group normalization accepts (no GPU): every product that 64 bits hold."""

import ctypes as C

import numpy as np
import pytest

from paper_2609_30846_amd import ipk
from workloads.generate import INT8, INT16


def _create(tin, tout, sw_qc, sw_q1, m_sw, shift_sw):
    g, c = np.full(64, 1 << 22, dtype=np.int32), np.zeros(64, dtype=np.int64)
    d = ipk.GroupNormDesc(64, 4, 1, 8, tin, tout, g.ctypes.data, c.ctypes.data, 25, 1, 1, sw_qc, sw_q1, m_sw, shift_sw)
    h = C.c_void_p()
    status = ipk.load().ipk_groupnorm_create(C.byref(d), C.byref(h))
    if status == ipk.IPK_OK:
        ipk.load().ipk_groupnorm_destroy(h)
    return status


@pytest.mark.parametrize("tin", [INT8, INT16])
@pytest.mark.parametrize("tout,shift_sw", [(INT8, 54), (INT16, 47)])
def test_multipliers_of_17_bits(tin, tout, shift_sw):
    """The polynomial on a grid of 2^-13: values of up to 2^45, so that 17-bit multipliers reach 2^62."""
    unit = 1 / 8192
    assert _create(tin, tout, int(2.4632 / unit), int(-1 / (0.1240 * unit * unit)) - 1, 130023,
                   shift_sw) not in (ipk.IPK_ERR_INVALID_ARG, ipk.IPK_ERR_UNSUPPORTED), ipk.last_error()


@pytest.mark.parametrize("m_sw,shift_sw,fits", [(131076, 33, True), (131076, 34, False), (131074, 48, True),
                                                (131074, 49, False)])
def test_the_limit_is_where_64_bits_end(m_sw, shift_sw, fits):
    """Swish(h) = 2^31 h for h > 0 with q_c = 0, q_1 = -2^30: its largest product is m_sw (2^46 - 2^31)."""
    assert (m_sw * (2 ** 46 - 2 ** 31) + 2 ** (shift_sw - 1) < 2 ** 63) == fits
    status = _create(INT16, INT16, 0, -(1 << 30), m_sw, shift_sw)
    if fits:
        assert status not in (ipk.IPK_ERR_INVALID_ARG, ipk.IPK_ERR_UNSUPPORTED), ipk.last_error()
    else:
        assert status == ipk.IPK_ERR_UNSUPPORTED and "2^63" in ipk.last_error()
