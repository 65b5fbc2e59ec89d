"""Limits of the microscaled calls that are refused before any device work."""

import ctypes as C

import pytest

from paper_2511_06724_amd import dn

P = 4096  # a 16-byte aligned address that is never followed


@pytest.mark.parametrize("N,K,msg", [(2 ** 22 + 32, 128, b"2^22"), (32, 2 ** 22 + 128, b"2^22"), (2 ** 18, 2 ** 17, b"too many values")])
def test_weights_past_the_products_limits_are_not_packed(N, K, msg):
    """The product takes N and K up to 2^22; a matrix of 2^35 values needs more threads than a launch has."""
    assert dn.lib.dn_pack_weight(dn.DN_MXFP4, P, N, K, P, None) == dn.DN_EINVAL
    assert msg in dn.lib.dn_last_error()
    if msg == b"2^22":
        n = C.c_int64(-7)
        assert dn.lib.dn_packed_weight_elems(dn.DN_MXFP4, N, K, C.byref(n)) == dn.DN_EINVAL and n.value == -7
