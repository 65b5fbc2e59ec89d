"""Argument checks of the microscaled entry points (no GPU: every case is refused before any
device work), and the sizes they report against the oracle's layout."""

import ctypes as C

import numpy as np
import pytest

from oracle import mx
from paper_2511_06724_amd import dn, workloads as W

P = 4096  # a 16-byte aligned address that is never followed
I63 = 2 ** 63 - 1


def _bytes(f, *args):
    n = C.c_int64(-7)
    return f(*args, C.byref(n)), n.value


@pytest.mark.parametrize("fmt", [dn.DN_MXFP4, dn.DN_MXFP8])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 32), (5, 33), (100000, 768), (2 ** 40, 64), (1, 2 ** 31 - 32)])
def test_bytes_match_the_oracle(fmt, rows, cols):
    assert dn.mx_bytes(fmt, rows, cols) == mx.n_bytes(fmt, rows, cols)


@pytest.mark.parametrize("args", [(dn.DN_FP8, 1, 1), (5, 1, 1), (dn.DN_MXFP4, 0, 1), (dn.DN_MXFP4, 1, 0), (dn.DN_MXFP8, -3, 4),
                                  (dn.DN_MXFP4, 1, 2 ** 31 - 31), (dn.DN_MXFP8, I63, 32), (dn.DN_MXFP4, 2 ** 47, 1)])
def test_bytes_refused(args):
    assert _bytes(dn.lib.dn_mx_bytes, *args) == (dn.DN_EINVAL, -7)


def test_null_size_outputs_refused():
    assert dn.lib.dn_mx_bytes(dn.DN_MXFP4, 1, 1, None) == dn.DN_EINVAL
    assert dn.lib.ac_mx_store_bytes(1, 1, None) == dn.DN_EINVAL
    assert dn.lib.ac_mx_lookup_bytes(1, 1, 1, None) == dn.DN_EINVAL


def test_store_workspace():
    assert dn.ac_mx_store_bytes(1, 10 ** 6) == 0
    assert dn.ac_mx_store_bytes(1000, 10 ** 6) == 4 * 10 ** 6
    for bad in ((0, 1), (1, 0), (-1, 5)):
        assert _bytes(dn.lib.ac_mx_store_bytes, *bad) == (dn.DN_EINVAL, -7)


QUANT = dict(dtype=dn.DN_MXFP4, src=dn.DN_BF16, x=P, ldx=64, rows=4, cols=64, q=P)


@pytest.mark.parametrize("change", [dict(dtype=dn.DN_BF16), dict(dtype=2), dict(src=dn.DN_FP8), dict(src=dn.DN_MXFP4), dict(x=None),
                                    dict(q=None), dict(ldx=63), dict(ldx=-64), dict(rows=0), dict(rows=2 ** 31), dict(cols=0),
                                    dict(cols=2 ** 31, ldx=2 ** 31), dict(q=P + 8), dict(x=P + 1), dict(src=dn.DN_FP32, x=P + 2)])
def test_quantize_refused(change):
    a = {**QUANT, **change}
    assert dn.lib.dn_mx_quantize(a["dtype"], a["src"], a["x"], a["ldx"], a["rows"], a["cols"], a["q"], None) == dn.DN_EINVAL
    assert dn.lib.dn_last_error()


@pytest.mark.parametrize("change", [dict(dtype=0), dict(q=None), dict(y=None), dict(ldy=63), dict(rows=-1), dict(q=P + 1)])
def test_dequantize_refused(change):
    a = {**dict(dtype=dn.DN_MXFP8, q=P, rows=4, cols=64, y=P, ldy=64), **change}
    assert dn.lib.dn_mx_dequantize(a["dtype"], a["q"], a["rows"], a["cols"], a["y"], a["ldy"], None) == dn.DN_EINVAL


STORE = dict(dtype=dn.DN_MXFP4, src=dn.DN_FP32, x=P, ldx=64, n=400, slots=P, table=P, n_slots=100, dim=64, ws=P)


@pytest.mark.parametrize("change", [dict(dtype=1), dict(src=4), dict(x=None), dict(slots=None), dict(table=None), dict(ws=None),
                                    dict(ws=P + 2), dict(ldx=32), dict(n=0), dict(n=2 ** 31), dict(n_slots=0), dict(dim=0),
                                    dict(table=P + 4)])
def test_store_refused(change):
    a = {**STORE, **change}
    assert dn.lib.ac_mx_store(a["dtype"], a["src"], a["x"], a["ldx"], a["n"], a["slots"], a["table"], a["n_slots"], a["dim"], a["ws"],
                              None) == dn.DN_EINVAL


@pytest.mark.parametrize("change", [dict(dtype=6), dict(table=None), dict(idx=None), dict(out=None), dict(n_slots=0), dict(n=0),
                                    dict(ldo=10), dict(dim=-1)])
def test_fetch_refused(change):
    a = {**dict(dtype=dn.DN_MXFP4, table=P, n_slots=5, dim=64, idx=P, n=3, out=P, ldo=64), **change}
    assert dn.lib.ac_mx_fetch(a["dtype"], a["table"], a["n_slots"], a["dim"], a["idx"], a["n"], a["out"], a["ldo"], None) == dn.DN_EINVAL


LOOKUP = dict(dtype=dn.DN_MXFP4, q=P, nq=3, table=P, n=100, dim=64, tab=None, idx=P, score=P, k=None, ws=P)


@pytest.mark.parametrize("change", [dict(dtype=0), dict(q=None), dict(table=None), dict(idx=None), dict(ws=None), dict(nq=0), dict(n=0),
                                    dict(dim=0), dict(dim=16385), dict(k=P), dict(tab=([0.5], [1, 2])), dict(ws=P + 8),
                                    dict(tab=([0.9, 0.5], [1, 2, 3]), k=P), dict(tab=([float("nan")], [1, 2]), k=P),
                                    dict(tab=([0.5], [3, 2]), k=P)])
def test_lookup_refused(change):
    a = {**LOOKUP, **change}
    tab = C.byref(dn.k_table(*a["tab"])) if a["tab"] else None
    assert dn.lib.ac_mx_lookup(a["dtype"], a["q"], a["nq"], a["table"], a["n"], a["dim"], tab, a["idx"], a["score"], a["k"], a["ws"],
                               None) == dn.DN_EINVAL


LINEAR = dict(dtype=dn.DN_MXFP4, x=P, w=P, bias=None, resid=None, rf=0, y=P, yf=0, M=4, N=64, K=128, geglu=0)


@pytest.mark.parametrize("change", [dict(dtype=dn.DN_MXFP8), dict(dtype=dn.DN_FP16), dict(x=None), dict(w=None), dict(y=None), dict(M=0),
                                    dict(M=2 ** 31), dict(N=48), dict(N=0), dict(K=64), dict(K=192), dict(K=0),
                                    dict(geglu=1, resid=P), dict(geglu=1, N=48), dict(geglu=1, N=2 ** 30), dict(x=P + 8), dict(w=P + 4),
                                    dict(geglu=1, y=P + 8), dict(y=P + 1), dict(yf=1, y=P + 2), dict(resid=P + 2, rf=1), dict(bias=P + 2)])
def test_linear_refused(change):
    a = {**LINEAR, **change}
    assert dn.lib.dn_op_linear(a["dtype"], a["x"], a["w"], a["bias"], a["resid"], a["rf"], a["y"], a["yf"], a["M"], a["N"], a["K"],
                               a["geglu"], None) == dn.DN_EINVAL


def test_pack_and_layernorm_refused():
    n = C.c_int64(-7)
    for N, K in ((48, 128), (64, 64), (0, 128)):
        assert dn.lib.dn_packed_weight_elems(dn.DN_MXFP4, N, K, C.byref(n)) == dn.DN_EINVAL and n.value == -7
        assert dn.lib.dn_pack_weight(dn.DN_MXFP4, P, N, K, P, None) == dn.DN_EINVAL
    assert dn.lib.dn_pack_weight(dn.DN_MXFP4, P, 64, 128, P + 8, None) == dn.DN_EINVAL
    assert dn.lib.dn_packed_weight_elems(dn.DN_MXFP8, 64, 128, C.byref(n)) == dn.DN_EINVAL
    for M, Cc, y in ((0, 64, P), (4, 36, P), (4, 64, P + 8), (4, 2080, P)):
        assert dn.lib.dn_op_layernorm(dn.DN_MXFP4, P, y, M, Cc, P, P, 1e-5, None) == dn.DN_EINVAL
    # other entry points take none of the new types
    assert dn.lib.dn_op_attention(dn.DN_MXFP4, P, 64, P, 64, P, 64, P, 64, 1, 1, 4, 4, 64, 0.1, None) == dn.DN_EINVAL
    assert dn.lib.dn_op_conv3x3(dn.DN_MXFP4, P, 1, 4, 4, 64, 0, 1, P, None, None, None, P, 8, 0, None) == dn.DN_EINVAL
    assert dn.lib.dn_op_layernorm_slabs(dn.DN_MXFP4, P, P, 4, 64, P, P, 1e-5, P, 2, None, 1, None) == dn.DN_EINVAL


def test_config():
    dn.weight_count(W.sdxl(W.DN_MXFP4))
    for bad in (W.sd15_level(W.DN_MXFP4), W.tiny(4), W.tiny(5)):   # 320-wide transformer; no such model types
        with pytest.raises(dn.DnError) as e:
            dn.weight_count(bad)
        assert e.value.code == dn.DN_EINVAL


def test_binding_checks_buffers_and_strides():
    import torch
    q = torch.zeros(mx.n_bytes(mx.MXFP4, 4, 64) - 1, dtype=torch.uint8)
    x = torch.zeros(4, 64)
    for f in (lambda: dn.mx_quantize(dn.DN_MXFP4, x, q, stream=0), lambda: dn.mx_quantize(dn.DN_MXFP4, x.t(), stream=0),
              lambda: dn.mx_quantize(dn.DN_MXFP4, x[0], stream=0), lambda: dn.mx_quantize(dn.DN_MXFP4, x.double(), stream=0),
              lambda: dn.mx_dequantize(dn.DN_MXFP4, q, 4, 64, stream=0),
              lambda: dn.ac_mx_store(dn.DN_MXFP4, x, torch.zeros(3, dtype=torch.int64), torch.zeros(9999, dtype=torch.uint8), 9, stream=0),
              lambda: dn.ac_mx_store(dn.DN_MXFP4, x, torch.zeros(4, dtype=torch.int32), torch.zeros(9999, dtype=torch.uint8), 9, stream=0),
              lambda: dn.ac_mx_fetch(dn.DN_MXFP4, torch.zeros(99, dtype=torch.uint8), 9, torch.zeros(4, dtype=torch.int64), x, stream=0)):
        with pytest.raises(ValueError):
            f()


def test_too_large_for_one_launch_refused():
    """More work than a launch has threads, and offsets in a tile's rows past 32 bits."""
    rows, cols = 2 ** 31 - 1, 320
    assert dn.lib.dn_mx_quantize(dn.DN_MXFP4, dn.DN_FP32, P, cols, rows, cols, P, None) == dn.DN_EINVAL
    assert dn.lib.dn_mx_dequantize(dn.DN_MXFP8, P, rows, cols, P, cols, None) == dn.DN_EINVAL
    for n, k in ((2 ** 22 + 32, 128), (32, 2 ** 22 + 128)):
        assert dn.lib.dn_op_linear(dn.DN_MXFP4, P, P, None, None, 0, P, 1, 1, n, k, 0, None) == dn.DN_EINVAL
