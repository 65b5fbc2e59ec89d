"""Rotary positions, norms of query and key heads with the rotation, and attention of packed sequences
against the fp64 oracle.

Tolerances. u is half a step of the output type relative to the value (fp32 2^-24, bf16 2^-8), w = 2^-24.
Rotation: sine and cosine are within 4 w, a product and a sum round once more each: 8 w (|a| + |b|), then u |y|.
Norm: a sum of squares of up to 256 values in groups of eight and a tree of five levels is within 13 w,
its root half of that; root, quotient and two products round: 16 w in all, on both values of a pair.
Attention: a score is a sum of dim products, within dim w sum|q k| scale; with the scaling and the difference
to the reference maximum, four roundings of a score, that is the relative error d of a probability (and
the exponential's own 2 w). bf16 probabilities round by u in the product. o = sum p v / sum p is then within
2 (d + u_p) + (keys + 4) w of sum p |v|, then u |o|."""

import numpy as np
import pytest
import torch

from oracle import packed as P
from paper_2511_06724_amd import dn
from tests.gpu_util import DEV, announce, host, tdtype
from tests.test_packed_cpu import turns

pytestmark = pytest.mark.gpu

W = 2.0 ** -24
U = {dn.DN_FP32: 2.0 ** -24, dn.DN_BF16: 2.0 ** -8}
TYPES = [dn.DN_FP32, dn.DN_BF16]


def heads(rng, rows, n, dim, dtype, pad=0, std=1.0):
    """A device tensor [rows, n, dim] (a slice of a wider one with `pad` heads behind) and its values."""
    t = torch.from_numpy(rng.normal(size=(rows, n + pad, dim)).astype(np.float32) * std).to(DEV).to(tdtype(dtype))[:, :n]
    return t, host(t)


def int_t(a, dtype=torch.int32):
    return torch.tensor(a, device=DEV, dtype=dtype)


def positions(rng, rows, axes, far=False):
    lo, hi = (-2 ** 31, 2 ** 31) if far else (-50, 5000)
    p = rng.integers(lo, hi, (rows, axes)).astype(np.int32)
    return torch.from_numpy(p).to(DEV), p


def rope_tol(x, freqs, pairing, ref, dtype, w=8):
    half = len(freqs)
    a = np.abs(x)
    first = slice(0, 2 * half, 2) if pairing == P.PAIRS else slice(0, half)
    second = slice(1, 2 * half, 2) if pairing == P.PAIRS else slice(half, 2 * half)
    s = a[..., first] + a[..., second]
    t = w * W * a
    t[..., first], t[..., second] = w * W * s, w * W * s
    return t + U[dtype] * np.abs(ref)


def close(got, ref, tol):
    assert np.isfinite(got).all() and (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) - tol).max())


ROPES = [(64, (32, 32), True), (128, (32, 48, 48), False), (80, (16, 24, 24), True), (128, (128,), True), (256, (256,), True),
         (8, (8,), True), (16, (2, 2, 2, 2), False), (96, (16, 40), True), (32, (8,), True), (200, (160,), False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", [dn.DN_ROPE_PAIRS, dn.DN_ROPE_HALVES])
@pytest.mark.parametrize("dim,axes,per_axis", ROPES)
def test_rope(dtype, pairing, dim, axes, per_axis):
    for rows, n, far in ((1, 1, True), (7, 5, False), (300, 13, True)):
        announce(f"rope {dtype} {pairing} {dim} {axes} {rows} x {n}")
        rng = np.random.default_rng(rows)
        x, xv = heads(rng, rows, n, dim, dtype, pad=1)
        pos, pv = positions(rng, rows, len(axes), far)
        table = dn.rope_table(axes, 10000.0, per_axis)
        freqs = dn.rope_freqs(axes, 10000.0, per_axis)
        ref = P.rotate(xv, pv, freqs, axes, pairing)
        y = dn.op_rope(x, pos, table, pairing=pairing)
        close(host(y), ref, rope_tol(xv, freqs, pairing, ref, dtype))
        # in place, on a strided tensor, and whatever lies behind it stays
        whole = x._base if x._base is not None else x
        behind = whole[:, n:].clone()
        dn.op_rope(x, pos, table, x, pairing=pairing)
        assert torch.equal(x, y) and torch.equal(whole[:, n:], behind)


def test_rope_backwards_and_large_grid():
    """Negated positions turn back; many rows take the variant of several heads a lane group."""
    rng = np.random.default_rng(5)
    x, xv = heads(rng, 9000, 9, 64, dn.DN_FP32)
    pos, pv = positions(rng, 9000, 2)
    table = dn.rope_table((32, 32))
    y = dn.op_rope(x, pos, table)
    ref = P.rotate(xv, pv, dn.rope_freqs((32, 32)), (32, 32), P.PAIRS)
    close(host(y), ref, rope_tol(xv, dn.rope_freqs((32, 32)), P.PAIRS, ref, dn.DN_FP32))
    back = dn.op_rope(y, -pos, table)
    assert (back - x).abs().max().item() <= 2 * 16 * W * 2 * x.abs().max().item()
    few = dn.op_rope(x[:5], pos[:5].contiguous(), table)
    assert torch.equal(few, y[:5])


def test_rope_gradient_is_the_inverse_rotation():
    """d/dx of <g, rotate(x)> is rotate(g) at the negated position, against differences of the (linear) call."""
    rng = np.random.default_rng(6)
    x, xv = heads(rng, 3, 2, 16, dn.DN_FP32)
    g, gv = heads(rng, 3, 2, 16, dn.DN_FP32)
    pos, _ = positions(rng, 3, 1)
    table = dn.rope_table((12,))
    grad = host(dn.op_rope(g, -pos, table))
    for at in ((0, 0, 0), (1, 1, 11), (2, 0, 15)):
        e = torch.zeros_like(x)
        e[at] = 1.0
        diff = (gv * host(dn.op_rope(e, pos, table))).sum()
        assert abs(diff - grad[at]) <= 40 * W * np.abs(gv).max()


def test_values_past_the_rotated_width_pass_whole():
    x = torch.randn(4, 3, 64, device=DEV)
    x[..., 32:] = torch.tensor([float("inf"), float("nan"), -float("inf"), 3.0], device=DEV).repeat(8)
    pos, _ = positions(np.random.default_rng(0), 4, 1, True)
    for pairing in (dn.DN_ROPE_PAIRS, dn.DN_ROPE_HALVES):
        y = dn.op_rope(x, pos, dn.rope_table((32,)), pairing=pairing)
        assert torch.equal(torch.nan_to_num(y[..., 32:], 7.0, 8.0, 9.0), torch.nan_to_num(x[..., 32:], 7.0, 8.0, 9.0))
        assert torch.isfinite(y[..., :32]).all()


@pytest.mark.parametrize("freq", [10.0, 100.0, 30000.3, -65536.0])
def test_rope_at_any_frequency(freq):
    """The angle of far positions, taken in integers: 2^-31 of a turn moves values of size one by 0.05 w, beside the rotation's
    own 8 w and the output's rounding."""
    pos = [2 ** 31 - 1, -2 ** 31, 1234567891, -7, 0]
    x = torch.zeros(len(pos), 1, 8, device=DEV)
    x[..., 0] = 1.0
    y = host(dn.op_rope(x, int_t([[p] for p in pos]), dn.rope_table((2,), freqs=[freq])))[:, 0]
    angle = [2 * np.pi * (p * turns(freq) % 2 ** 64) / 2.0 ** 64 for p in pos]
    close(y[:, 0], np.cos(angle), 9.05 * W)
    close(y[:, 1], np.sin(angle), 9.05 * W)
    assert not y[:, 2:].any()


# ----------------------------------------------------------------------------- norm and rotation

def norm_rope_ref(xv, gain, eps, pv, freqs, axes, pairing, dtype):
    n = P.rms_norm(xv, gain, eps)
    ref = P.rotate(n, pv, freqs, axes, pairing)
    return ref, rope_tol(n, freqs, pairing, ref, dtype, w=24)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", [dn.DN_ROPE_PAIRS, dn.DN_ROPE_HALVES])
@pytest.mark.parametrize("dim,axes,per_axis", ROPES)
def test_qk_norm_rope(dtype, pairing, dim, axes, per_axis):
    for rows, hq, hk, with_v in ((1, 1, 1, False), (6, 5, 1, True), (130, 8, 2, True), (1500, 20, 4, True)):
        announce(f"qk_norm_rope {dtype} {pairing} {dim} {rows} x {hq}, {hk}")
        rng = np.random.default_rng(rows + dim)
        qkv = torch.from_numpy(rng.normal(size=(rows, hq + 2 * hk, dim)).astype(np.float32) * 3).to(DEV).to(tdtype(dtype))
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        gq, gk = (torch.from_numpy(rng.normal(1, 0.3, dim).astype(np.float32)).to(DEV) for _ in range(2))
        pos, pv = positions(rng, rows, len(axes))
        table, freqs = dn.rope_table(axes, 5e5, per_axis), dn.rope_freqs(axes, 5e5, per_axis)
        qo, ko, vo = (torch.full((rows, h, dim), 7.0, device=DEV, dtype=qkv.dtype) for h in (hq, hk, hk))
        before = qkv.clone()
        dn.op_qk_norm_rope(q, k, gq, gk, 1e-6, pos, table, qo, ko, v if with_v else None, vo if with_v else None, pairing=pairing)
        assert torch.equal(qkv, before)
        for x, g, o in ((q, gq, qo), (k, gk, ko)):
            ref, tol = norm_rope_ref(host(x), host(g), 1e-6, pv, freqs, axes, pairing, dtype)
            close(host(o), ref, tol)
        assert torch.equal(vo, v if with_v else torch.full_like(vo, 7.0))
        # in place
        dn.op_qk_norm_rope(q, k, gq, gk, 1e-6, pos, table, q, k, pairing=pairing)
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(v, before[:, hq + hk:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 64, 128, 200])
def test_norm_of_large_and_tiny_heads(dtype, dim):
    """Heads whose squares leave 32 bits, up to the largest and down to the smallest values of a type: scaling by powers of two
    is exact, so the bound is the same."""
    rng = np.random.default_rng(dim)
    axes, rows = (8,), 9
    table, freqs = dn.rope_table(axes), dn.rope_freqs(axes)
    gain = torch.from_numpy(rng.normal(1, 0.3, dim).astype(np.float32)).to(DEV)
    pos, pv = positions(rng, rows, 1)
    for size in (1e38, 1e25, 3e19, 1e18, 1.0, 1e-11, 1e-13, 1e-18, 1e-25, 1e-36) + ((3e-43,) if dtype == dn.DN_FP32 else ()):
        x = torch.from_numpy((rng.uniform(0.5, 3, (rows, 3, dim)) * rng.choice([-1, 1], (rows, 3, dim)) * size).astype(np.float32)).to(DEV)
        x[0] = 0
        x[0, :, dim // 2] = size                         # one value alone
        x[1, :, 1::2] = 1e-3                             # sizes of many kinds
        x = x.to(tdtype(dtype))
        for eps in (0.0, 1e-40, 1e-22, 1e-6, 1e30, 3e38):
            announce(f"norm {dtype} {dim} {size} {eps}")
            q, k = torch.empty_like(x[:, :2]), torch.empty_like(x[:, 2:])
            dn.op_qk_norm_rope(x[:, :2], x[:, 2:], gain, gain, eps, pos, table, q, k)
            ref, tol = norm_rope_ref(host(x), host(gain), float(np.float32(eps)), pv, freqs, axes, P.PAIRS, dtype)
            close(host(torch.cat([q, k], 1)), ref, tol + 2.0 ** -130)    # (an output below 2^-126 has fewer bits)
    # infinities and NaN as the formula has them
    x = torch.ones(2, 1, dim, device=DEV, dtype=tdtype(dtype))
    x[0, 0, 3], x[1, 0, 5] = float("inf"), float("nan")
    q, k, zero = torch.empty_like(x), torch.empty_like(x), torch.zeros(2, 1, device=DEV, dtype=torch.int32)
    dn.op_qk_norm_rope(x, x, gain, gain, 1e-6, zero, dn.rope_table((2,)), q, k)
    assert torch.isnan(q[0, 0, 3]) and (q[0, 0, 4:] == 0).all() and torch.isnan(q[1]).all()


def cache_rows(q_len, kv_start, kv_len):
    return [kv_start[s] + kv_len[s] - n + i for s, n in enumerate(q_len) for i in range(n)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_len", [[1], [1] * 70, [0, 3, 0, 0, 17, 1, 0], [5, 64, 2]])
def test_qk_norm_rope_into_a_cache(dtype, q_len):
    rng = np.random.default_rng(len(q_len))
    dim, hq, hk, axes = 64, 4, 2, (24, 16)
    n, total = len(q_len), sum(q_len)
    kv_len = [m + int(rng.integers(0, 9)) for m in q_len]
    order, at, kv_start = rng.permutation(n), 0, [0] * n
    for s in order:                                          # sequences lie in the cache in another order, with gaps
        at += int(rng.integers(0, 3))
        kv_start[s] = at
        at += kv_len[s]
    rows = at + 5
    extra = 3                                                # packed rows behind the last sequence
    q, qv = heads(rng, total + extra, hq, dim, dtype)
    k, kv = heads(rng, total + extra, hk, dim, dtype, pad=1)
    v, vv = heads(rng, total + extra, hk, dim, dtype)
    gain = torch.ones(dim, device=DEV)
    pos, pv = positions(rng, total + extra, 2)
    table, freqs = dn.rope_table(axes), dn.rope_freqs(axes)
    qo = torch.full((total + extra, hq, dim), 7.0, device=DEV, dtype=q.dtype)
    kc, vc = (torch.full((rows, hk, dim), 9.0, device=DEV, dtype=q.dtype) for _ in range(2))
    seqs = dn.Sequences(int_t(np.cumsum([0] + q_len)), int_t(kv_start, torch.int64), int_t(kv_len), max(max(kv_len), 1))
    dn.op_qk_norm_rope(q, k, gain, gain, 1e-6, pos, table, qo, kc, v, vc, seqs)
    ref, tol = norm_rope_ref(qv, 1.0, 1e-6, pv, freqs, axes, P.PAIRS, dtype)
    close(host(qo[:total]), ref[:total], tol[:total])
    assert (qo[total:] == 7).all()
    ref, tol = norm_rope_ref(kv, 1.0, 1e-6, pv, freqs, axes, P.PAIRS, dtype)
    to = cache_rows(q_len, kv_start, kv_len)
    close(host(kc)[to], ref[:total], tol[:total])
    assert np.array_equal(host(vc)[to], vv[:total])
    rest = np.setdiff1d(np.arange(rows), to)
    assert (kc[rest] == 9).all() and (vc[rest] == 9).all()


BAD = [  # (q_start, kv_start, kv_len) of three sequences of 4 rows in a cache of 40, the bad one
    ([0, 4, 8, 12], [0, 37, 20], [4, 4, 4], 1), ([0, 4, 8, 12], [0, -1, 20], [4, 4, 4], 1), ([0, 4, 8, 12], [0, 10, 20], [4, -4, 4], 1),
    ([0, 4, 8, 12], [0, 2 ** 62, 20], [4, 4, 4], 1), ([0, 4, 8, 2 ** 31 - 1], [0, 10, 20], [4, 4, 4], 2),
    ([0, 4, 8, 12], [0, 10, 2 ** 63 - 1], [4, 4, 2 ** 31 - 1], 2), ([-5, 4, 8, 12], [0, 10, 20], [9, 4, 4], 0)]


@pytest.mark.parametrize("q_start,kv_start,kv_len,bad", BAD)
def test_sequences_outside_the_tensors_are_skipped(q_start, kv_start, kv_len, bad):
    rng = np.random.default_rng(3)
    seqs = dn.Sequences(int_t(q_start), int_t(kv_start, torch.int64), int_t(kv_len), 40)
    q, qv = heads(rng, 12, 4, 64, dn.DN_BF16)
    k, _ = heads(rng, 12, 2, 64, dn.DN_BF16)
    kc, kcv = heads(rng, 40, 2, 64, dn.DN_BF16)
    vc, vcv = heads(rng, 40, 2, 64, dn.DN_BF16)
    good = [s for s in range(3) if s != bad]
    o = torch.full_like(q, 7.0)
    ws = workspace(q, kc, seqs)
    dn.op_attention_packed(q, kc, vc, o, seqs, ws=ws)
    for s in range(3):
        part = host(o[4 * s:4 * s + 4])
        if s == bad:
            assert (part == 7).all()
            continue
        a = kv_start[s]
        ref, m = P.attention(qv[4 * s:4 * s + 4], kcv[a:a + 4], vcv[a:a + 4], True, 0.125)
        close(part, ref, 0.1 * m + 0.01)
    gain, table, pos = torch.ones(64, device=DEV), dn.rope_table((64,)), int_t([[i] for i in range(12)])
    before, qo = kc.clone(), torch.full_like(q, 7.0)
    dn.op_qk_norm_rope(q, k, gain, gain, 1e-6, pos, table, qo, kc, seqs=seqs)
    changed = {int(i) for i in (kc != before).flatten(1).any(1).nonzero()}
    assert changed == {kv_start[s] + i for s in good for i in range(4)}
    assert (qo[4 * bad:4 * bad + 4] == 7).all() and all((qo[4 * s:4 * s + 4] != 7).any() for s in good)


@pytest.mark.parametrize("q_start", [[4, 0, 8, 2], [12, 3, 1, 0], [0, 9, 5, 12], [2 ** 31 - 1, -5, 7, 2 ** 31 - 1]])
def test_starts_out_of_order_stay_in_bounds(q_start):
    """Not a promised input: nothing outside the tensors is read or written (poison around the outputs stays)."""
    n = 12
    for kv_len, bound in (([4, 4, 4], 40), ([40, 12, 6], 4000)):
        seqs = dn.Sequences(int_t(q_start), int_t([0, 10, 20], torch.int64), int_t(kv_len), bound)
        q, kv = torch.randn(n, 4, 64, device=DEV, dtype=torch.bfloat16), torch.randn(60, 2, 64, device=DEV, dtype=torch.bfloat16)
        whole, cache = torch.full((n + 200, 4, 64), 7.0, device=DEV, dtype=q.dtype), torch.full((460, 2, 64), 7.0, device=DEV, dtype=q.dtype)
        o, kc = whole[100:100 + n], cache[200:260]
        dn.op_attention_packed(q, kv, kv, o, seqs, ws=workspace(q, kv, seqs))
        pos, gain = torch.zeros(n, 1, device=DEV, dtype=torch.int32), torch.ones(64, device=DEV)
        dn.op_qk_norm_rope(q, kv[:n], gain, gain, 1e-6, pos, dn.rope_table((64,)), o, kc, seqs=seqs)
        assert (whole[:100] == 7).all() and (whole[100 + n:] == 7).all() and (cache[:200] == 7).all() and (cache[260:] == 7).all()


# ----------------------------------------------------------------------------- attention

def workspace(q, k, seqs):
    return torch.full((dn.attention_packed_bytes(q, k, seqs),), 0xff, device=DEV, dtype=torch.uint8)


class Batch:
    """A packed batch with gaps between the sequences' key rows that hold NaN, and packed rows behind the last one."""

    def __init__(self, q_len, kv_len, hq, hk, dim, dtype, seed=0, std=2.0, max_kv=None, behind=2):
        rng = np.random.default_rng(seed)
        self.q_len, self.kv_len, self.dtype = q_len, kv_len, dtype
        n, at, self.start = len(q_len), 1, [0] * len(q_len)
        for s in rng.permutation(n):
            self.start[s] = at
            at += kv_len[s] + int(rng.integers(0, 4))
        self.total = sum(q_len)
        self.q, self.qv = heads(rng, self.total + behind, hq, dim, dtype, pad=1, std=std)
        kv = torch.full((at + 1, 2 * hk, dim), float("nan"), device=DEV, dtype=tdtype(dtype))
        for s in range(n):
            kv[self.start[s]:self.start[s] + kv_len[s]] = torch.from_numpy(
                rng.normal(size=(kv_len[s], 2 * hk, dim)).astype(np.float32)).to(DEV).to(tdtype(dtype))
        self.k, self.v = kv[:, :hk], kv[:, hk:]
        self.o = torch.full((self.total + behind, hq, dim), 7.0, device=DEV, dtype=tdtype(dtype))
        self.qs = np.cumsum([0] + q_len)
        self.seqs = dn.Sequences(int_t(self.qs), int_t(self.start, torch.int64), int_t(kv_len), max_kv or max(max(kv_len), 1))
        self.scale = dim ** -0.5
        self.ws = workspace(self.q, self.k, self.seqs)

    def run(self, causal, scale=None, stream=None):
        dn.op_attention_packed(self.q, self.k, self.v, self.o, self.seqs, causal=causal, scale=scale, ws=self.ws, stream=stream)
        return self.o

    def expect(self, causal, scale=None, rows=None):
        """(packed rows, reference, tolerance) of every sequence (of its rows `rows`)."""
        kv, vv = host(self.k), host(self.v)
        dim = kv.shape[-1]
        scale = self.scale if scale is None else scale
        up = U[self.dtype] if self.dtype == dn.DN_BF16 else 0.0
        for s, (n, m) in enumerate(zip(self.q_len, self.kv_len)):
            a, b = self.qs[s], self.start[s]
            q, k, v = self.qv[a:a + n], kv[b:b + m], vv[b:b + m]
            pick = np.arange(n) if rows is None else np.unique(np.clip(rows, 0, max(n - 1, 0)))[:n]
            ref, mass = (np.zeros((n,) + self.qv.shape[1:]) for _ in range(2))
            for i in pick:
                seen = min(m, max(0, m - n + i + 1)) if causal else m
                ref[i], mass[i] = (t[0] for t in P.attention(q[i:i + 1], k[:seen], v[:seen], False, scale))
            if m and n:
                size = max(np.abs(q).sum(-1).max() * np.abs(k).max(), 1e-30) * abs(scale)
                d = (dim + 4) * W * size + 2 * W
            else:
                d = 0.0
            tol = (2 * (d + up) + (m + 4) * W) * mass + U[self.dtype] * np.abs(ref)
            yield a + pick, ref[pick], tol[pick]

    def check(self, causal, scale=None, rows=None):
        got = host(self.o)
        for at, ref, tol in self.expect(causal, scale, rows):
            close(got[at], ref, tol)
        assert (self.o[self.total:] == 7).all(), "packed rows behind the last sequence"


LENGTHS = [([1], [1]), ([1], [77]), ([63, 1, 64], [63, 1, 64]), ([65, 129, 2], [65, 130, 300]), ([0, 5, 0, 33, 0], [0, 5, 9, 64, 0]),
           ([7, 3, 40], [3, 0, 39]), ([1] * 67, list(range(0, 134, 2)))]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hk,dim", [(2, 2, 64), (8, 2, 128), (5, 1, 64), (3, 3, 32), (8, 1, 96), (4, 2, 128)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", range(len(LENGTHS)))
def test_attention(dtype, hq, hk, dim, causal, lengths):
    q_len, kv_len = LENGTHS[lengths]
    announce(f"attention {dtype} {hq}/{hk} x {dim} {causal} {q_len[:5]} {kv_len[:5]}")
    b = Batch(q_len, kv_len, hq, hk, dim, dtype, seed=lengths)
    b.run(causal)
    b.check(causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_len,kv_len,hq,hk,dim", [([700], [700], 4, 1, 128), ([513, 20], [900, 1500], 2, 2, 64),
                                                    ([1, 1, 2], [5000, 20, 1300], 8, 2, 128), ([3], [9000], 6, 2, 64),
                                                    ([600, 600], [600, 600], 2, 2, 128)])
def test_attention_long(dtype, q_len, kv_len, hq, hk, dim):
    for causal in (True, False):
        announce(f"long attention {dtype} {q_len} {kv_len} {causal}")
        b = Batch(q_len, kv_len, hq, hk, dim, dtype, seed=9)
        first = b.run(causal).clone()
        b.check(causal, rows=np.array([0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 300, 511, 512, 598, 599, 698, 699]))
        assert torch.equal(b.run(causal), first), "the same inputs, the same bits"


# One batch for every way a call is run: tiles of 2, 4 and 8 waves, units of 32 rows whole and divided, by lengths and heads.
WAYS = [(dn.DN_BF16, 128, [40, 90, 33], [40, 90, 33], 3, 3), (dn.DN_BF16, 64, [70, 1, 50], [200, 80, 50], 4, 2),
        (dn.DN_BF16, 96, [40, 60], [41, 77], 2, 1), (dn.DN_BF16, 32, [90, 20], [90, 400], 2, 2),
        (dn.DN_BF16, 128, [300, 129], [300, 400], 4, 4), (dn.DN_BF16, 64, [450, 2], [500, 2], 2, 2),
        (dn.DN_BF16, 96, [320, 190], [330, 190], 1, 1), (dn.DN_BF16, 32, [257, 200], [257, 260], 4, 2),
        (dn.DN_BF16, 128, [1030, 1100], [1030, 1500], 52, 52), (dn.DN_BF16, 128, [130], [3000], 8, 1), (dn.DN_BF16, 64, [60, 64], [2000, 900], 2, 2),
        (dn.DN_FP32, 64, [40, 300], [40, 900], 4, 2), (dn.DN_FP32, 128, [200], [1800], 4, 2), (dn.DN_FP32, 96, [1030, 900], [1100, 900], 8, 8),
        (dn.DN_FP32, 32, [1000], [1000], 20, 20), (dn.DN_FP32, 128, [1000, 1], [1000, 70], 16, 16), (dn.DN_FP32, 64, [700, 800], [720, 800], 12, 12)]


@pytest.mark.parametrize("way", range(len(WAYS)))
@pytest.mark.parametrize("causal", [True, False])
def test_attention_each_way(way, causal):
    dtype, dim, q_len, kv_len, hq, hk = WAYS[way]
    announce(f"way {way}: {dtype} {dim} {q_len} {kv_len} {hq}/{hk} {causal}")
    b = Batch(q_len, kv_len, hq, hk, dim, dtype, seed=way)
    first = b.run(causal).clone()
    b.check(causal, rows=np.array([0, 1, 17, 31, 32, 63, 64, 100, 127, 128, 255, 256, 300, 1029, 1099]))
    assert torch.equal(b.run(causal), first)
    # values that are not finite, in the last key of the last sequence: no other sequence or earlier row sees it
    m = kv_len[-1]
    b.v[b.start[-1] + m - 1] = float("nan")
    b.run(causal)
    last = b.total - 1
    assert torch.isnan(b.o[last]).all()
    b.v[b.start[-1] + m - 1] = 0.0
    for s, (at, ref, tol) in enumerate(b.expect(causal, rows=np.array([0, 1, 31, 200]))):
        if s < len(q_len) - 1:
            close(host(b.o)[at], ref, tol)
        elif causal:
            keep = at < last
            close(host(b.o)[at[keep]], ref[keep], tol[keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,m,group", [(300, 300, 1), (1, 300, 4), (130, 1000, 2), (9, 2500, 8), (1, 20000, 1)])
def test_every_key_counts_once(dtype, dim, n, m, group):
    """Equal scores: a row's output is the share of its keys with every value; one key too few or too many shows."""
    b = Batch([n], [m], group, 1, dim, dtype)
    b.q.zero_()
    b.qv[:] = 0
    b.v[b.start[0]:b.start[0] + m] = 0
    b.v[b.start[0] + torch.arange(m, device=DEV), 0, torch.arange(m, device=DEV) % dim] = 1
    got = host(b.run(True))[:n]
    for i in range(n):
        seen = m - n + i + 1
        share = np.bincount(np.arange(seen) % dim, minlength=dim) / seen
        # p = 1 exactly; the sum is exact below 2^24 keys: one quotient and the output round
        assert (np.abs(got[i] - share) <= (2 * W + U[dtype]) * share).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,group", [(64, 1), (128, 4), (32, 2), (96, 1)])
def test_masked_keys_have_no_influence(dtype, dim, group):
    """Infinities and NaN in keys and values that a row does not see (the later tokens of its own sequence) leave it alone;
    a row that sees them gets what the formula gives."""
    n = 150
    b = Batch([n, 40], [n, 40], 2 * group, 2, dim, dtype, seed=2)
    clean, want = host(b.run(True)), list(b.expect(True))
    a = b.start[0]
    b.k[a + 100] = float("nan")
    b.k[a + 120, :, ::2] = float("inf")
    b.v[a + 90, 0, :] = float("inf")
    b.v[a + 95, 0, 3] = -float("inf")
    b.v[a + 97, 1, 5] = float("nan")
    got = host(b.run(True))
    h0, h1 = slice(0, group), slice(group, 2 * group)
    # A run that meets them adds in another order: what stays finite is within the tolerance of the formula again.
    (_, ref, tol), (_, ref2, tol2) = want
    close(clean[:n], ref, tol)
    close(got[:90], ref[:90], tol[:90])
    close(got[n:n + 40], ref2, tol2)
    assert (got[90:95, h0] == np.inf).all()
    close(got[90:97, h1], ref[90:97, h1], tol[90:97, h1])
    assert np.isnan(got[95:100, h0, 3]).all() and (got[95:100, h0, 4:] == np.inf).all()
    assert np.isnan(got[97:100, h1, 5]).all()
    close(got[97:100, h1, 6:], ref[97:100, h1, 6:], tol[97:100, h1, 6:])
    assert np.isnan(got[100:n]).all() and (b.o[n + 40:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m,hq,hk,dim", [(1, 100, 2, 2, 64), (1, 4000, 2, 2, 64), (1, 60000, 1, 1, 64), (130, 3000, 8, 1, 128),
                                           (300, 700, 2, 2, 128), (40, 90, 3, 3, 32), (1, 9000, 8, 1, 96)])
@pytest.mark.parametrize("first", [True, False])
def test_an_infinite_value_of_little_weight(dtype, n, m, hq, hk, dim, first):
    """Its weight is e^-300 of the sum, zero in 32 bits: the row's value is infinite all the same, wherever the key lies."""
    b = Batch([n], [m], hq, hk, dim, dtype)
    b.q.zero_()
    b.q[..., 0] = 1.0
    a, last = b.start[0], b.start[0] + m - n
    low, high = (a + 1, last) if first else (last, a + 1)
    b.k[a:a + m, :, 0] = 0.0
    b.k[high, :, 0] = 300.0
    b.v[low, :, 3], b.v[low, :, 5], b.v[low, :, 7] = float("inf"), -float("inf"), float("nan")
    got = host(b.run(True, scale=1.0))[:n]
    want = host(b.v[high]).repeat(hq // hk, 0)
    assert (got[..., 3] == np.inf).all() and (got[..., 5] == -np.inf).all() and np.isnan(got[..., 7]).all()
    assert np.array_equal(got[..., 8:], np.broadcast_to(want[:, 8:], got[..., 8:].shape))


def test_extreme_scores():
    """Scores of +-1e30 and equal ones at the lowest finite value: the largest take all, no NaN."""
    b = Batch([4], [70], 1, 1, 64, dn.DN_FP32)
    a = b.start[0]
    b.q.fill_(1.0)
    b.k[a:a + 70] = -1e28
    b.k[a + 3] = 1e28
    b.run(False, scale=1.0)
    assert torch.allclose(b.o[:4], b.v[a + 3].expand(4, 1, 64))
    b.k[a:a + 70] = -1e28                                      # every score -6.4e29: the mean
    b.run(False, scale=1.0)
    assert torch.allclose(b.o[:4], b.v[a:a + 70].mean(0).expand(4, 1, 64), atol=1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("longest,q_max", [(150, 1), (3000, 1), (900, 6), (400, 130)])
def test_many_sequences(dtype, longest, q_max):
    """More sequences than a wave has lanes, among them empty ones."""
    rng = np.random.default_rng(longest)
    q_len = [int(n) for n in rng.integers(0, q_max + 1, 211)]
    kv_len = [n + int(m) for n, m in zip(q_len, rng.integers(0, longest - q_max, 211))]
    b = Batch(q_len, kv_len, 4, 2, 64, dtype, seed=5)
    b.run(True)
    b.check(True, rows=np.array([0, 1, 5, 31, 32, 70, 129]))


def test_a_shared_prefix():
    """Sequences whose keys overlap: all of them begin with the same rows."""
    for dtype in TYPES:
        b = Batch([1] * 5 + [40], [1200, 1100, 700, 1, 1200, 1199], 8, 2, 128, dtype)
        b.start = [b.start[0]] * 6
        b.seqs = dn.Sequences(int_t(b.qs), int_t(b.start, torch.int64), int_t(b.kv_len), 1200)
        b.run(True)
        b.check(True, rows=np.arange(0, 40, 13))


@pytest.mark.parametrize("dtype", TYPES)
def test_offsets_past_32_bits(dtype):
    """Keys and values that lie 4 GiB and more behind the tensors' starts, inside one sequence and at its start."""
    rng, hk, dim, width = np.random.default_rng(2), 2, 64, 1024
    rows = 2 ** 32 // (width * dim * (2 if dtype == dn.DN_BF16 else 4)) + 4000
    kv = torch.empty(rows, width, dim, device=DEV, dtype=tdtype(dtype))
    k, v = kv[:, :hk], kv[:, hk:2 * hk]
    kv[:, :2 * hk].normal_(generator=torch.Generator(device=DEV).manual_seed(3))
    tail = rows - 1500
    kh, vh = host(k.contiguous()), host(v.contiguous())
    for q_len, kv_len, start in (([1, 1], [rows, 1500], [0, tail]), ([2000, 300], [rows, 1500], [0, tail])):
        q, qv = heads(rng, sum(q_len), 4, dim, dtype)
        o = torch.empty_like(q)
        seqs = dn.Sequences(int_t(np.cumsum([0] + q_len)), int_t(start, torch.int64), int_t(kv_len), rows)
        dn.op_attention_packed(q, k, v, o, seqs, causal=False, ws=workspace(q, k, seqs))
        got, up = host(o), U[dtype] if dtype == dn.DN_BF16 else 0.0
        for s in range(2):
            for i in {0, q_len[s] - 1}:
                at, a, m = i + s * q_len[0], start[s], kv_len[s]
                ref, mass = P.attention(qv[at:at + 1], kh[a:a + m], vh[a:a + m], False, dim ** -0.5)
                d = (dim + 4) * W * np.abs(qv[at]).sum(-1).max() * np.abs(kh).max() * dim ** -0.5 + 2 * W
                close(got[at:at + 1], ref, (2 * (d + up) + (m + 4) * W) * mass + U[dtype] * np.abs(ref))
    # the last rows of the cache are written
    x, gain = heads(rng, 3, hk, dim, dtype)[0], torch.ones(dim, device=DEV)
    seqs = dn.Sequences(int_t([0, 3]), int_t([tail], torch.int64), int_t([1500]), rows)
    near = (torch.empty(3, hk, dim, device=DEV, dtype=x.dtype) for _ in range(2))
    args = (x, x, gain, gain, 1e-6, int_t([[5], [6], [7]]), dn.rope_table((dim,)))
    qo, ko = near
    dn.op_qk_norm_rope(*args, qo, k, x, v, seqs)
    dn.op_qk_norm_rope(*args, qo, ko)
    assert torch.equal(k[-3:], ko) and torch.equal(v[-3:], x)


def test_the_longest_keys():
    """As many keys as are counted, equal scores: first, middle and last ones have their weights. More are skipped."""
    torch.cuda.empty_cache()
    rows, most = 2 ** 31 - 1, 2 ** 31 - 65537
    if torch.cuda.mem_get_info()[0] < rows * 64 + 2 ** 30:
        pytest.skip("137 GB of keys")
    kv = torch.zeros(rows, 1, 32, device=DEV, dtype=torch.bfloat16)
    kv[0], kv[2 ** 30 + 5], kv[most - 1] = 1.0, 2.0, 4.0
    kv[most:] = 8.0
    q = torch.zeros(3, 1, 32, device=DEV, dtype=torch.bfloat16)
    for causal in (True, False):
        o = torch.full_like(q, 7.0)
        seqs = dn.Sequences(int_t([0, 1, 2, 3]), int_t([0, 0, most - 1], torch.int64), int_t([most, rows, 2]), most)
        dn.op_attention_packed(q, kv, kv, o, seqs, causal=causal, ws=workspace(q, kv, seqs))
        got = host(o)
        # parts of 2^21 keys or so are exact, their sum rounds 1024 times
        assert (np.abs(got[0] * most / 7 - 1) <= U[dn.DN_BF16] + 1030 * W).all() and (got[1] == 7).all() and (got[2] == 6).all()
    del kv
    torch.cuda.empty_cache()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(scale):
    for dtype in TYPES:
        b = Batch([70, 1], [90, 33], 4, 2, 64, dtype, seed=4, std=1.0)
        b.run(True, scale=scale)
        b.check(True, scale=scale)


@pytest.mark.parametrize("bound", [1, 100, 100000])
def test_the_bound_of_the_lengths_decides_no_result(bound):
    b = Batch([1, 5], [3000, 777], 8, 2, 128, dn.DN_BF16, max_kv=bound)
    b.run(True)
    b.check(True)


def test_a_captured_call_follows_lengths_and_data():
    """Capture once; replay with the lengths, keys and queries of the moment, with eager work between."""
    b = Batch([1, 1, 1], [40, 300, 2000], 8, 2, 128, dn.DN_BF16)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b.run(True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.run(True)
    kv_len = b.seqs._keep[2]
    for lens in ([40, 300, 2000], [39, 1, 1999], [0, 300, 64]):
        kv_len.copy_(int_t(lens))
        b.kv_len = lens
        b.o.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.check(True)
        replayed = b.o.clone()
        b.ws.fill_(0xff)
        assert torch.equal(b.run(True), replayed)


def test_a_captured_step_generates():
    """Norm, rotation into the cache and attention of one token per request, captured together with the work that moves
    positions and lengths on: replayed, with eager calls between, it gives the eager steps' bits."""
    hq, hk, dim, cap = 4, 2, 64, 700
    gen = torch.Generator(device=DEV).manual_seed(4)
    new = [torch.empty(3, hq + 2 * hk, dim, device=DEV, dtype=torch.bfloat16).normal_(generator=gen) for _ in range(4)]
    table, gain = dn.rope_table((dim,)), torch.ones(dim, device=DEV)

    def state():
        kv_len = int_t([600, 0, 33])
        seqs = dn.Sequences(int_t([0, 1, 2, 3]), int_t([0, cap, 2 * cap], torch.int64), kv_len, cap)
        kc, vc = (torch.zeros(3 * cap, hk, dim, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        kc.normal_(generator=torch.Generator(device=DEV).manual_seed(6))
        vc.normal_(generator=torch.Generator(device=DEV).manual_seed(7))
        x = torch.empty_like(new[0])
        q, o = (torch.empty(3, hq, dim, device=DEV, dtype=x.dtype) for _ in range(2))
        return dict(kv_len=kv_len, seqs=seqs, kc=kc, vc=vc, x=x, q=q, o=o, pos=int_t([[599], [-1], [32]]), ws=workspace(q, kc, seqs))

    def step(s):
        s["kv_len"].add_(1)
        s["pos"].add_(1)
        x = s["x"]
        dn.op_qk_norm_rope(x[:, :hq], x[:, hq:hq + hk], gain, gain, 1e-6, s["pos"], table, s["q"], s["kc"], x[:, hq + hk:], s["vc"], s["seqs"])
        dn.op_attention_packed(s["q"], s["kc"], s["vc"], s["o"], s["seqs"], ws=s["ws"])

    a, b = state(), state()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(b)
    for x in new:
        a["x"].copy_(x)
        b["x"].copy_(x)
        step(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a["o"], b["o"]) and torch.equal(a["kc"], b["kc"]) and torch.equal(a["vc"], b["vc"])
        assert torch.equal(a["kv_len"], b["kv_len"]) and torch.isfinite(a["o"]).all() and (a["o"] != 0).any()


def test_tensors_of_another_device_are_refused():
    b = Batch([1], [9], 2, 2, 64, dn.DN_BF16)
    with pytest.raises(ValueError, match="current GPU"):
        dn.op_attention_packed(b.q, b.k.cpu(), b.v, b.o, b.seqs)
    with pytest.raises(ValueError, match="current GPU"):
        dn.op_rope(b.q, torch.zeros(len(b.q), 1, dtype=torch.int32), dn.rope_table((64,)))


def test_the_last_token_of_a_long_projection():
    """One row whose stride is more than rows may lie apart, and no multiple of 16 bytes."""
    width, rows = 3 * 4 * 64 + 1, 11000
    whole = torch.randn(1, rows, width, device=DEV).to(torch.bfloat16)
    at = (rows - 1) * width // 8 * 8                   # 16-byte aligned
    x = whole.flatten()[at:][:768].view(12, 64).as_strided((1, 12, 64), (rows * width, 64, 1))
    q, k, v = x[:, :4], x[:, 4:8], x[:, 8:]
    assert q.stride(0) > 2 ** 23
    pos, gain, table = int_t([[rows]]), torch.ones(64, device=DEV), dn.rope_table((64,))
    qo, ko, vo, qc, kc, vc = (torch.empty(1, 4, 64, device=DEV, dtype=x.dtype) for _ in range(6))
    dn.op_qk_norm_rope(q, k, gain, gain, 1e-6, pos, table, qo, ko, v, vo)
    dn.op_qk_norm_rope(q.contiguous(), k.contiguous(), gain, gain, 1e-6, pos, table, qc, kc, v.contiguous(), vc)
    assert torch.equal(qo, qc) and torch.equal(ko, kc) and torch.equal(vo, vc) and torch.equal(v, vo)
    assert torch.equal(dn.op_rope(q, pos, table), dn.op_rope(q.contiguous(), pos, table))


@pytest.mark.parametrize("raw", [False, True])
def test_new_tensors_of_a_call_on_another_stream(raw):
    """Their memory is not what the current stream has freed and still writes."""
    other = torch.cuda.Stream()
    on = other.cuda_stream if raw else other
    x, _ = heads(np.random.default_rng(0), 4096, 8, 64, dn.DN_FP32)
    m = x.reshape(4096, 512)
    pos, w = torch.arange(4096, device=DEV, dtype=torch.int32)[:, None].contiguous(), torch.randn(512, 1024, device=DEV)
    table = dn.rope_table((64,))
    want = dn.op_rope(x, pos, table)
    q = dn.mx_quantize(dn.DN_MXFP8, m)
    deq, packed = dn.mx_dequantize(dn.DN_MXFP8, q, 4096, 512), dn.pack_weight(dn.DN_FP32, w, 512, 1024)
    busy = torch.randn(8192, 8192, device=DEV)
    calls = [(want, lambda: dn.op_rope(x, pos, table, stream=on)), (table.data, lambda: dn.rope_table((64,), stream=on).data),
             (q, lambda: dn.mx_quantize(dn.DN_MXFP8, m, stream=on)), (packed, lambda: dn.pack_weight(dn.DN_FP32, w, 512, 1024, stream=on)),
             (deq, lambda: dn.mx_dequantize(dn.DN_MXFP8, q, 4096, 512, stream=on))]
    for expect, call in calls:
        torch.cuda.synchronize()
        for _ in range(4):
            torch.mm(busy, busy)                        # some milliseconds
        freed = torch.empty_like(expect)
        freed.fill_(3)
        del freed
        got = call()
        other.synchronize()
        torch.cuda.synchronize()
        n = 4096 * (512 + 16) if expect is q else None      # (what follows the scales is never written)
        assert torch.equal(got[:n], expect[:n])


def test_two_streams_at_once():
    bs = [Batch([1, 3], [2500, 1200], 8, 2, 128, dn.DN_BF16, seed=s) for s in (1, 2)]
    want = [b.run(True).clone() for b in bs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in bs]
    for _ in range(20):
        for b, s in zip(bs, streams):
            b.run(True, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(b.o, w) for b, w in zip(bs, want))


# ----------------------------------------------------------------------------- the layer

@pytest.mark.parametrize("dtype", TYPES)
def test_layer_prompt_then_tokens(dtype):
    """Norm and rotation into the cache, then attention over it, as a server runs them: a prompt in one call gives what
    the same prompt gives in a chunk and single tokens, and both match the oracle."""
    rng = np.random.default_rng(8)
    dim, hq, hk, axes, lens = 64, 4, 2, (16, 24, 24), [9, 70]
    cap, total = 96, sum(lens)
    table, freqs = dn.rope_table(axes, 1e4), dn.rope_freqs(axes, 1e4)
    qkv, vals = heads(rng, total, hq + 2 * hk, dim, dtype)
    gq, gk = (torch.from_numpy(rng.normal(1, 0.2, dim).astype(np.float32)).to(DEV) for _ in range(2))
    pos, pv = positions(rng, total, 3)

    def step(rows, q_len, kv_len, kc, vc):
        x, p = qkv[rows].contiguous(), pos[rows].contiguous()
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        seqs = dn.Sequences(int_t(np.cumsum([0] + q_len)), int_t([0, cap], torch.int64), int_t(kv_len), cap)
        qo, o = (torch.empty(len(rows), hq, dim, device=DEV, dtype=x.dtype) for _ in range(2))
        dn.op_qk_norm_rope(q, k, gq, gk, 1e-6, p, table, qo, kc, v, vc, seqs)
        dn.op_attention_packed(qo, kc, vc, o, seqs, ws=workspace(qo, kc, seqs))
        return o

    cache = [torch.zeros(2 * cap, hk, dim, device=DEV, dtype=qkv.dtype) for _ in range(4)]
    whole = step(list(range(total)), lens, lens, cache[0], cache[1])
    parts = torch.empty_like(whole)
    done = [0, 0]
    for n in ([5, 66], [1, 1], [1, 1], [1, 1], [1, 0], [0, 1]):
        rows = [done[0] + i for i in range(n[0])] + [lens[0] + done[1] + i for i in range(n[1])]
        done = [done[0] + n[0], done[1] + n[1]]
        parts[rows] = step(rows, n, done, cache[2], cache[3])
    assert done == lens
    assert torch.equal(cache[0], cache[2]) and torch.equal(cache[1], cache[3])
    q = P.rotate(P.rms_norm(vals[:, :hq], host(gq), 1e-6), pv, freqs, axes, P.PAIRS)
    k = P.rotate(P.rms_norm(vals[:, hq:hq + hk], host(gk), 1e-6), pv, freqs, axes, P.PAIRS)
    for s, a in enumerate((0, lens[0])):
        ref, mass = P.attention(q[a:a + lens[s]], k[a:a + lens[s]], vals[a:a + lens[s], hq + hk:], True, dim ** -0.5)
        # q and k round by u, so a score by 2 u |q||k| scale at most; the rest as above
        size = np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max() * dim ** -0.5
        d = 2 * U[dtype] * size + (dim + 32) * W * size * dim ** 0.5
        tol = (2 * (d + U[dtype]) + 80 * W) * mass + U[dtype] * np.abs(ref)
        close(host(whole[a:a + lens[s]]), ref, tol)
        close(host(parts[a:a + lens[s]]), ref, tol)
