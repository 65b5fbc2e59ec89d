"""Argument checks of the packed-sequence entry points (no GPU: every case is refused before any device work)."""

import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2511_06724_amd import dn
from tests.test_epilogue_cpu import HIPCC, ROOT

P = 4096  # a 16-byte aligned address that is never followed


def seqs(**change):
    a = {**dict(n=2, max_kv_len=64, q_start=P, kv_start=P, kv_len=P), **change}
    return C.byref(dn._Sequences(a["n"], a["max_kv_len"], a["q_start"], a["kv_start"], a["kv_len"]))


def rot(**change):
    a = {**dict(table=P, pos=P, n_axes=2, rot_dim=64, pairing=0), **change}
    return dn._rotation_bytes(a["table"] or 0, a["pos"] or 0, a["n_axes"], a["rot_dim"], a["pairing"])


BAD_SEQS = [dict(n=0), dict(n=-1), dict(max_kv_len=0), dict(q_start=None), dict(kv_start=None), dict(kv_len=None), dict(q_start=P + 2),
            dict(kv_start=P + 4), dict(kv_len=P + 1)]
BAD_ROT = [dict(table=None), dict(pos=None), dict(table=P + 8), dict(pos=P + 2), dict(n_axes=0), dict(n_axes=5), dict(rot_dim=0),
           dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=-2), dict(pairing=2), dict(pairing=-1), dict(pairing=1, rot_dim=60)]


@pytest.mark.parametrize("freqs,dims", [([0.5], [3]), ([0.5], [0]), ([0.5], [-2]), ([float("nan")], [2]), ([float("inf")], [2]),
                                        ([65537.0], [2]), ([0.5] * 129, [258]), ([0.5] * 129, [130, 128])])
def test_rope_table_refused(freqs, dims):
    f, d = np.array(freqs, np.float64), np.array(dims, np.int32)
    assert dn.lib.dn_rope_table(f.ctypes.data, d.ctypes.data, len(dims), P, None) == dn.DN_EINVAL
    assert dn.lib.dn_last_error()


def test_rope_table_pointers_refused():
    f, d = np.array([0.5]), np.array([2], np.int32)
    for args in ((None, d.ctypes.data, 1, P), (f.ctypes.data, None, 1, P), (f.ctypes.data, d.ctypes.data, 1, None),
                 (f.ctypes.data, d.ctypes.data, 1, P + 8), (f.ctypes.data, d.ctypes.data, 0, P), (f.ctypes.data, d.ctypes.data, 5, P)):
        assert dn.lib.dn_rope_table(*args, None) == dn.DN_EINVAL


ROPE = dict(dtype=dn.DN_BF16, x=P, ldx=128, y=P + 64, ldy=128, T=4, heads=2, dim=64, rot=rot())


@pytest.mark.parametrize("change", [dict(dtype=dn.DN_FP8), dict(dtype=dn.DN_FP16), dict(x=None), dict(y=None), dict(x=P + 8), dict(ldx=120),
                                    dict(ldx=132), dict(ldy=127), dict(T=0), dict(T=2 ** 31), dict(heads=0), dict(heads=3), dict(dim=60),
                                    dict(dim=0), dict(dim=264, ldx=528, ldy=528), dict(rot=None), dict(y=P, ldx=136),
                                    dict(dtype=dn.DN_FP32, ldx=130)] + [dict(rot=rot(**b)) for b in BAD_ROT])
def test_rope_refused(change):
    a = {**ROPE, **change}
    assert dn.lib.dn_op_rope(a["dtype"], a["x"], a["ldx"], a["y"], a["ldy"], a["T"], a["heads"], a["dim"], a["rot"], None) == dn.DN_EINVAL


QKN = dict(dtype=dn.DN_BF16, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, T=4, heads=4, kv_heads=2, dim=64, gq=P, gk=P, eps=1e-6, rot=rot(),
           seqs=seqs(), qo=P + 64, ldqo=256, ko=P + 64, ldko=128, vo=P + 64, ldvo=128, rows=100)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(q=None), dict(k=None), dict(v=None), dict(vo=None), dict(qo=None), dict(ko=None),
                                    dict(ldq=248), dict(ldk=120), dict(ldv=100), dict(ldqo=192), dict(ldko=64), dict(ldvo=64), dict(T=0),
                                    dict(heads=0), dict(kv_heads=0), dict(dim=12), dict(gq=None), dict(gk=None), dict(gq=P + 2), dict(eps=-1.0),
                                    dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=0), dict(ko=P), dict(vo=P),
                                    dict(qo=P, ldqo=264), dict(seqs=None, ko=P, ldko=136), dict(seqs=None, vo=P, ldvo=136), dict(k=P + 2),
                                    dict(vo=P + 4), dict(rows=2 ** 41)]
                         + [dict(rot=rot(**b)) for b in BAD_ROT] + [dict(seqs=seqs(**b)) for b in BAD_SEQS])
def test_qk_norm_rope_refused(change):
    a = {**QKN, **change}
    assert dn.lib.dn_op_qk_norm_rope(a["dtype"], a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["T"], a["heads"], a["kv_heads"],
                                     a["dim"], a["gq"], a["gk"], a["eps"], a["rot"], a["seqs"], a["qo"], a["ldqo"], a["ko"], a["ldko"],
                                     a["vo"], a["ldvo"], a["rows"], None) == dn.DN_EINVAL


ATTN = dict(dtype=dn.DN_BF16, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, o=P + 64, ldo=256, T=4, rows=100, heads=4, kv_heads=2, dim=64, seqs=seqs(),
            causal=1, scale=0.125, ws=P)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(dtype=5), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=P + 8),
                                    dict(ldq=248), dict(ldk=64), dict(ldv=124), dict(ldo=0), dict(T=0), dict(T=2 ** 31), dict(T=2 ** 30),
                                    dict(rows=0), dict(rows=2 ** 41), dict(heads=0), dict(heads=5), dict(kv_heads=0), dict(kv_heads=3),
                                    dict(dim=48), dict(dim=256, ldq=1024, ldk=512, ldv=512, ldo=1024), dict(seqs=None), dict(causal=2),
                                    dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-3e38),
                                    dict(o=P), dict(ws=P + 8)] + [dict(seqs=seqs(**b)) for b in BAD_SEQS])
def test_attention_packed_refused(change):
    a = {**ATTN, **change}
    assert dn.lib.dn_op_attention_packed(a["dtype"], a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["o"], a["ldo"], a["T"], a["rows"],
                                         a["heads"], a["kv_heads"], a["dim"], a["seqs"], a["causal"], a["scale"], a["ws"], None) == dn.DN_EINVAL


@pytest.mark.parametrize("args", [(2, 4, 4, 2, 64, 2, 64), (1, 0, 4, 2, 64, 2, 64), (1, 4, 4, 3, 64, 2, 64), (1, 4, 4, 2, 80, 2, 64),
                                  (1, 4, 4, 2, 64, 0, 64), (1, 4, 4, 2, 64, 2, 0), (1, 2 ** 31, 4, 2, 64, 2, 64)])
def test_workspace_size_refused(args):
    n = C.c_int64(-7)
    assert dn.lib.dn_attention_packed_bytes(*args, C.byref(n)) == dn.DN_EINVAL and n.value == -7
    assert dn.lib.dn_attention_packed_bytes(1, 4, 4, 2, 64, 2, 64, None) == dn.DN_EINVAL


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_other_types_and_shapes():
    i32, i64 = torch.int32, torch.int64
    good = dict(q_start=t(3, dtype=i32), kv_start=t(2, dtype=i64), kv_len=t(2, dtype=i32))
    s = dn.Sequences(**good, max_kv_len=9)
    for change in (dict(q_start=t(2, dtype=i32)), dict(kv_start=t(2, dtype=i32)), dict(kv_len=t(2, dtype=i64)), dict(kv_len=t(2, 1, dtype=i32)),
                   dict(q_start=t(6, dtype=i32)[::2])):
        with pytest.raises(ValueError):
            dn.Sequences(**{**good, **change}, max_kv_len=9)
    qkv = dict(q=t(5, 4, 64), k=t(9, 2, 64), v=t(9, 2, 64), o=t(5, 4, 64))
    for change in (dict(q=t(5, 4, 64, dtype=torch.float16)), dict(k=t(9, 2, 64, dtype=torch.float32)), dict(v=t(8, 2, 64)), dict(o=t(5, 4, 32)),
                   dict(q=t(5, 256)), dict(k=t(9, 2, 32), v=t(9, 2, 32)), dict(q=t(5, 64, 4).transpose(1, 2)), dict(q=t(5, 4, 128)[..., ::2])):
        with pytest.raises(ValueError):
            dn.op_attention_packed(**{**qkv, **change}, seqs=s, stream=0)


def test_binding_refuses_positions_and_gains():
    class Table:
        n_axes, rot_dim, address = 2, 64, P
    x = t(5, 4, 64)
    for pos in (t(5, 2), t(5, 3, dtype=torch.int32), t(4, 2, dtype=torch.int32), t(5, 4, dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            dn.op_rope(x, pos, Table, stream=0)
    pos, g = t(5, 2, dtype=torch.int32), t(64, dtype=torch.float32)
    good = dict(q=x, k=t(5, 2, 64), q_gain=g, k_gain=g, q_out=t(5, 4, 64), k_out=t(5, 2, 64))
    for change in (dict(q_gain=t(64)), dict(k_gain=t(32, dtype=torch.float32)), dict(k=t(4, 2, 64)), dict(k_out=t(6, 2, 64)), dict(k_out=t(5, 4, 64)),
                   dict(q_out=t(5, 4, 64, dtype=torch.float32)), dict(v=t(5, 2, 64)), dict(v=t(5, 4, 64), v_out=t(5, 2, 64))):
        with pytest.raises(ValueError):
            dn.op_qk_norm_rope(**{**good, **change}, eps=1e-6, pos=pos, table=Table, stream=0)


def test_binding_refuses_host_tensors():
    class Table:
        n_axes, rot_dim, address, device = 2, 64, P, -1
    i32 = torch.int32
    s = dn.Sequences(t(3, dtype=i32), t(2, dtype=torch.int64), t(2, dtype=i32), 9)
    q, k, pos, g = t(5, 4, 64), t(9, 2, 64), t(5, 2, dtype=i32), t(64, dtype=torch.float32)
    for call in (lambda: dn.op_rope(q, pos, Table, stream=0), lambda: dn.op_attention_packed(q, k, k, q, s, stream=0),
                 lambda: dn.op_qk_norm_rope(q, k[:5], g, g, 1e-6, pos, Table, q, k, k[:5], k, s, stream=0),
                 lambda: dn.rope_table((32, 32), device="cpu", stream=0)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


@pytest.mark.parametrize("stride", [0, 3, 100, 256, 2 ** 24, 2 ** 40])
def test_a_single_row_has_any_stride(stride):
    x = t(256).as_strided((1, 4, 64), (stride, 64, 1))
    assert dn._heads(x, "x")[1] == 256
    assert dn._heads(t(512).as_strided((2, 4, 64), (256, 64, 1)), "x")[1] == 256


def test_default_frequencies():
    assert dn.rope_freqs((4, 4), 100.0) == [1.0, 0.1, 1.0, 0.1]
    assert np.allclose(dn.rope_freqs((4, 4), 100.0, per_axis=False), 100.0 ** (-np.arange(4) / 4))
    with pytest.raises(ValueError):
        dn.RopeTable((4,), [1.0], "cpu", stream=0)


def turns(freq):
    """freq / (2 pi) modulo 1 in units of 2^-64, rounded, in integers (pi by Machin's formula in 400 bits)."""
    one = 1 << 400

    def arctan_of_inverse(x):
        total, term, n = 0, one // x, 1
        while term:
            total += term // n if n % 4 == 1 else -(term // n)
            term //= x * x
            n += 2
        return total

    two_pi = 8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239))
    num, den = float(freq).as_integer_ratio()
    return ((2 * num * one << 64) // (den * two_pi) + 1) // 2 % 2 ** 64


@pytest.mark.parametrize("freq", [1.0, 10.0, 100.0, 30000.3, 65536.0, 65535.99999999999, 2 * np.pi, -3.7, -65536.0, 0.123, 1e-6, 2.0 ** -70,
                                  -2.0 ** -63, 1e-300, 5e-324, 0.0])
def test_turns_of_a_frequency(freq):
    """The table's 64-bit turns per position are the nearest: 2^31 positions are off by 2^-34 of a turn, whatever the frequency."""
    f = dn.lib["_ZN2dn9rope_turnEd"]
    f.argtypes, f.restype = [C.c_double], C.c_uint64
    off = (f(freq) - turns(freq)) % 2 ** 64
    assert min(off, 2 ** 64 - off) <= 1


ATTENDS = r"""
#include "packed.h"
#include <cstdio>
int main() {
  const int most = 0x7fffffff;
  const long long rows = 1ll << 40;
  struct { int a, b; long long T; int len; long long k0, rows; bool want; } c[] = {
    {0, 1, 1, 0, 0, 1, true}, {0, 1, 1, 1, 0, 1, true}, {0, 1, 1, 1, 1, 1, false}, {0, 1, 1, 2, 0, 1, false}, {1, 1, 9, 1, 0, 9, false},
    {-1, 1, 9, 1, 0, 9, false}, {2, 1, 9, 1, 0, 9, false}, {0, 10, 9, 1, 0, 9, false}, {0, 1, 1, -1, 0, 9, false}, {0, 1, 1, 1, -1, 9, false},
    {0, 1, 1, most - 65536, 0, rows, true}, {0, 1, 1, most - 65535, 0, rows, false}, {0, 1, 1, most, 0, rows, false},
    {0, 1, 1, most - 65536, rows - most + 65536, rows, true}, {0, 1, 1, most - 65536, rows - most + 65537, rows, false},
    {0, 1, 1, 5, 0x7fffffffffffffffll, rows, false}, {most - 1, most, most, 5, 0, 5, true}, {0, most, most - 1, 5, 0, 5, false}};
  for (const auto& x : c)
    if (dn::sequence_attends(x.a, x.b, x.T, x.len, x.k0, x.rows) != x.want)
      return std::printf("%d %d %lld %d %lld %lld\n", x.a, x.b, x.T, x.len, x.k0, x.rows), 1;
  // a tile past the last key is still a number of 32 bits
  int end;
  return __builtin_add_overflow(dn::kMaxKeys, 65536, &end);
}
"""


@pytest.mark.skipif(HIPCC is None, reason="no hipcc")
def test_sequences_that_attention_takes(tmp_path):
    """The check of a sequence's rows and lengths, compiled for the host: inside the tensors, keys counted in 32 bits."""
    src, exe = tmp_path / "attends.hip", tmp_path / "attends"
    src.write_text(ATTENDS)
    r = subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I",
                        os.path.join(ROOT, "paper_2511_06724_amd", "csrc"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
