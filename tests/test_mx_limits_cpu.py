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


@pytest.mark.parametrize("off", [1, 2, 4])
def test_buffers_off_their_elements_refused(off):
    """Every buffer of the row calls is aligned to its elements: fp32 rows 4 bytes, slots and indices 8."""
    f = dn.DN_MXFP4
    calls = [lambda: dn.lib.ac_mx_store(f, dn.DN_FP32, P, 64, 4, P + off, P, 9, 64, None, None),
             lambda: dn.lib.ac_mx_fetch(f, P, 9, 64, P + off, 4, P, 64, None),
             lambda: dn.lib.ac_mx_lookup(f, P, 3, P, 9, 64, None, P + off, P, None, P, None)]
    if off < 4:
        tab = C.byref(dn.k_table([0.5], [1, 2]))
        calls += [lambda: dn.lib.dn_mx_dequantize(f, P, 4, 64, P + off, 64, None),
                  lambda: dn.lib.ac_mx_fetch(f, P, 9, 64, P, 4, P + off, 64, None),
                  lambda: dn.lib.ac_mx_lookup(f, P, 3, P, 9, 64, None, P, P + off, None, P, None),
                  lambda: dn.lib.ac_mx_lookup(f, P, 3, P, 9, 64, tab, P, P, P + off, P, None)]
    if off < 2:
        calls += [lambda: dn.lib.ac_mx_lookup(f, P + off, 3, P, 9, 64, None, P, P, None, P, None)]
    for call in calls:
        assert call() == dn.DN_EINVAL
        assert b"misaligned" in dn.lib.dn_last_error()


def test_store_workspace_of_more_slots_than_a_table_has_refused():
    n = C.c_int64(-7)
    assert dn.lib.ac_mx_store_bytes(1000, 2 ** 62, C.byref(n)) == dn.DN_EINVAL and n.value == -7
    assert dn.lib.ac_mx_store_bytes(1000, 2 ** 46, C.byref(n)) == dn.DN_OK and n.value == 2 ** 48


@pytest.mark.parametrize("dtype", [dn.DN_FP32, dn.DN_BF16, dn.DN_FP8, dn.DN_MXFP4])
@pytest.mark.parametrize("M", [2 ** 26 - 3, 2 ** 40])
def test_more_rows_than_a_layernorm_launch_has_refused(dtype, M):
    assert dn.lib.dn_op_layernorm(dtype, P, P, M, 32, P, P, 1e-5, None) == dn.DN_EINVAL
    assert b"one launch" in dn.lib.dn_last_error()


@pytest.mark.parametrize("change", [dict(score="float64"), dict(score="int32"), dict(k="float32"), dict(k="int64"), dict(idx="float64")])
def test_lookup_outputs_of_another_type_refused(change):
    import torch
    t = {**dict(idx="int64", score="float32", k="int32"), **change}
    out = [torch.zeros(4, dtype=getattr(torch, t[n])) for n in ("idx", "score", "k")]
    table, ws = (torch.zeros(n, dtype=torch.uint8) for n in (dn.mx_bytes(dn.DN_MXFP4, 9, 64), dn.ac_mx_lookup_bytes(4, 9, 64)))
    with pytest.raises(ValueError):
        dn.ac_mx_lookup(dn.DN_MXFP4, torch.zeros(4, 64, dtype=torch.float16), table, 9, ws, *out, [0.5], [1, 2], stream=0)
