"""Microscaled rows on the GPU against the oracle (oracle.mx, 64 bits): quantisation and reading
back bit for bit, the cache calls, the 4-bit product, the 4-bit LayerNorm, the search over a
quantised table, and runs of them together: on other streams, in captured graphs, in the
denoiser.

Tolerances. fp32 sums of K exact products differ from the exact sum by at most (K + 2) 2^-24 times
the sum of the magnitudes (the bias and the residual count as two more terms); a bf16 output
adds 2^-8 of the value (half its epsilon). GELU is within 4e-7 |g| (1.5e-7 of the erf formula, half
of it times |g|; 2^-22 for the exponential and the reciprocal) and its slope is below 1.13."""

import numpy as np
import pytest
import torch

from oracle import layers as L, mx, sampler, schedule as S, unet
from paper_2511_06724_amd import dn, workloads as W
from tests.gpu_util import DEV, announce, f32_dev, host, rel_l2

pytestmark = pytest.mark.gpu

FMTS = [dn.DN_MXFP4, dn.DN_MXFP8]
TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


def _rng(*seed):
    return np.random.default_rng(list(seed))


def _u8(n, fill=0xAA):
    return torch.full((n,), fill, device=DEV, dtype=torch.uint8)


def _wide(r, rows, cols):
    """Normal rows whose blocks differ in size, with blocks of zeros and of large values."""
    x = r.standard_normal((rows, cols))
    return x * 2.0 ** r.integers(-3, 4, (rows, -(-cols // 32))).repeat(32, 1)[:, :cols]


def _special(x, t):
    """Puts infinities, NaN, the type's extremes, subnormals, zeros and ties into the rows."""
    x = torch.from_numpy(np.ascontiguousarray(x)).to(t).clone()
    f = torch.finfo(t)
    flat = x.view(-1)
    put = [(0, float("inf")), (33, float("nan")), (70, f.min), (101, f.max), (133, f.tiny), (165, f.tiny / 4), (197, -0.0)]
    for i, v in put:
        if i < flat.numel():
            flat[i] = v
    if x.shape[1] >= 512:
        x[0, 256:288] = 0
        x[0, 288:320] = torch.tensor([4.0] + [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25] * 3 + [7.5]).to(t)
        x[0, 320:352] = f.tiny / 8
    return x


# ----------------------------------------------------------------------------- quantisation

@pytest.mark.parametrize("rows,cols,pad,off", [(1, 1, 0, 0), (3, 33, 0, 0), (5, 31, 2, 1), (2, 64, 0, 0), (7, 2100, 4, 0),
                                              (64, 768, 0, 0), (300, 100, 28, 3), (2, 70001, 0, 0), (3000, 32, 0, 0)])
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_bitwise(fmt, t, rows, cols, pad, off):
    announce(f"quantize fmt={fmt} {t} {rows}x{cols} stride +{pad} offset {off}")
    x = _special(_wide(_rng(rows, cols, fmt), rows, cols), t)
    store = torch.full((off + rows * (cols + pad),), float("nan"), dtype=t)
    view = store[off:].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    dev = store.to(DEV)[off:].view(rows, cols + pad)[:, :cols]
    q = _u8(dn.mx_bytes(fmt, rows, cols))
    dn.mx_quantize(fmt, dev, q)
    got = q.cpu().numpy()
    c, s = mx.quantize(x.double().numpy(), fmt)
    want = mx.to_buffer(c, s, fmt)
    assert np.array_equal(got[:want.size], want)
    assert (got[want.size:] == 0xAA).all()
    # and back, into rows of another stride: nothing is written beside them
    y = torch.full((rows, cols + 5), 7.0, device=DEV)
    dn.mx_dequantize(fmt, q, rows, cols, y[:, :cols])
    y = y.cpu().numpy()
    assert (y[:, cols:] == 7.0).all()
    with np.errstate(invalid="ignore"):
        assert np.array_equal(y[:, :cols], mx.values(c, s, fmt, cols).astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("fmt", FMTS)
def test_every_code_at_every_scale_reads_back(fmt):
    announce(f"all codes x all scales, fmt={fmt}")
    per = 16 if fmt == dn.DN_MXFP4 else 256
    codes = np.tile(np.arange(per, dtype=np.uint8), (256, 32 // 16 if per == 16 else 1))
    s = np.repeat(np.arange(256, dtype=np.uint8)[:, None], codes.shape[1] // 32, 1)
    buf = np.zeros(dn.mx_bytes(fmt, 256, codes.shape[1]), np.uint8)
    b = mx.to_buffer(codes, s, fmt)
    buf[:b.size] = b
    y = dn.mx_dequantize(fmt, torch.from_numpy(buf).to(DEV), 256, codes.shape[1]).cpu().numpy()
    assert np.array_equal(y, mx.values(codes, s, fmt, codes.shape[1]).astype(np.float32), equal_nan=True)


# ----------------------------------------------------------------------------- the cache

@pytest.mark.parametrize("n,n_slots,dim", [(1, 3, 2100), (7, 5, 33), (32, 64, 768), (33, 20, 64), (1000, 400, 100), (17000, 30000, 32)])
@pytest.mark.parametrize("fmt", FMTS)
def test_store_and_fetch(fmt, n, n_slots, dim):
    """Slots occur twice (the last row wins), lie outside the table (skipped), or are untouched."""
    announce(f"store/fetch fmt={fmt} n={n} slots={n_slots} dim={dim}")
    r = _rng(n, n_slots, dim)
    x = torch.from_numpy(_wide(r, n, dim)).to(torch.bfloat16)
    slots = r.integers(-2, n_slots + 2, n)
    if n > 2:
        slots[-1] = slots[0] = n_slots - 1
        slots[1] = 2 ** 40
    old = _wide(r, n_slots, dim)
    table = dn.mx_quantize(fmt, f32_dev(old))
    ws = _u8(max(dn.ac_mx_store_bytes(n, n_slots), 1), 0x5C)
    dn.ac_mx_store(fmt, x.to(DEV), torch.from_numpy(slots).to(DEV), table, n_slots, ws)
    want = mx.rounded(old.astype(np.float32), fmt)
    new = mx.rounded(x.double().numpy(), fmt)
    for j in range(n):
        if 0 <= slots[j] < n_slots:
            want[slots[j]] = new[j]
    got = host(dn.mx_dequantize(fmt, table, n_slots, dim))
    assert np.array_equal(got, want)
    idx = r.integers(-2, n_slots + 2, 50)
    out = torch.full((50, dim + 3), -3.0, device=DEV)
    dn.ac_mx_fetch(fmt, table, n_slots, torch.from_numpy(idx).to(DEV), out[:, :dim])
    out = host(out)
    for j in range(50):
        ok = 0 <= idx[j] < n_slots
        assert np.array_equal(out[j, :dim], want[idx[j]] if ok else np.full(dim, -3.0))
    assert (out[:, dim:] == -3.0).all()


# a workgroup's share of one row, of two and of many; whole words of scales and single ones; the most rows whose
# slots workgroups compare by themselves, and one more
@pytest.mark.parametrize("n,n_slots,dim", [(5, 9, 65536), (3, 4, 4097), (64, 70, 5120), (200, 90, 128), (255, 300, 32), (256, 120, 1),
                                           (256, 40, 2560), (257, 130, 64), (600, 650, 777)])
@pytest.mark.parametrize("fmt", FMTS)
def test_store_and_fetch_shapes(fmt, n, n_slots, dim):
    test_store_and_fetch(fmt, n, n_slots, dim)


def test_fetch_and_store_rows_at_any_element():
    """Sources and targets whose rows begin at every element of a 16-byte word, of every type."""
    announce("mx rows at odd addresses")
    r = _rng(77)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        for cols in (8, 61, 256):
            for off in range(8):
                x = torch.from_numpy(r.standard_normal((9, cols + off)).astype(np.float32)).to(dt)
                dev = torch.zeros(off + x.numel(), device=DEV, dtype=dt)[off:].view(9, cols + off).copy_(x)[:, :cols]
                want = mx.rounded(x[:, :cols].double().numpy(), mx.MXFP8)
                table = _u8(dn.mx_bytes(dn.DN_MXFP8, 9, cols), 0)
                dn.ac_mx_store(dn.DN_MXFP8, dev, torch.arange(9, device=DEV), table, 9)
                out = torch.full((off + 9 * (cols + off),), 2.5, device=DEV)
                view = out[off:].view(9, cols + off)[:, :cols]
                dn.ac_mx_fetch(dn.DN_MXFP8, table, 9, torch.arange(8, -1, -1, device=DEV), view)
                assert np.array_equal(host(view), want[::-1])
                view.fill_(2.5)
                assert (host(out) == 2.5).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_tables_past_32_bits(fmt):
    """Slots whose codes begin past 2^32 bytes: stored, read back and (as embeddings) found."""
    dim = 1024
    n = (1 << 32) // (dim // 2 if fmt == dn.DN_MXFP4 else dim) + 1000
    announce(f"table of {n} x {dim}, fmt={fmt}: {dn.mx_bytes(fmt, n, dim) >> 20} MB")
    table = torch.zeros(dn.mx_bytes(fmt, n, dim), device=DEV, dtype=torch.uint8)
    x = torch.from_numpy(_rng(3).standard_normal((3, dim)).astype(np.float32)).to(DEV)
    slots = torch.tensor([n - 1, 5, n - 500], device=DEV)
    dn.ac_mx_store(fmt, x, slots, table, n)
    out = torch.empty(3, dim, device=DEV)
    dn.ac_mx_fetch(fmt, table, n, slots, out)
    assert np.array_equal(host(out), mx.rounded(x.cpu().numpy(), fmt))
    for nq in (1, 9):
        q = torch.cat([x, x, x])[:nq].half().contiguous()
        idx, score = torch.empty(nq, device=DEV, dtype=torch.int64), torch.empty(nq, device=DEV)
        dn.ac_mx_lookup(fmt, q, table, n, _u8(dn.ac_mx_lookup_bytes(nq, n, dim)), idx, score)
        assert idx.tolist() == [n - 1, 5, n - 500] * (nq // 3) if nq == 9 else idx.tolist() == [n - 1]
        assert (score > 0.98).all()
    del table
    torch.cuda.empty_cache()


# ----------------------------------------------------------------------------- the product

def _interleave(w):
    n = w.shape[0] // 2
    return np.stack([w[:n].reshape(n // 32, 32, -1), w[n:].reshape(n // 32, 32, -1)], 1).reshape(2 * n, *w.shape[1:])


def _operands(r, M, Nw, K):
    x = _wide(r, M, K).astype(np.float32)
    w = (_wide(r, Nw, K) / np.sqrt(K)).astype(np.float32)
    b = r.standard_normal(Nw).astype(np.float32)
    return x, w, b, mx.rounded(x, mx.MXFP4), mx.rounded(w, mx.MXFP4)


def _matmul(a, b):
    return (torch.from_numpy(a).to(DEV) @ torch.from_numpy(b).to(DEV).t()).cpu().numpy()


# each row tile and column tile whole, one short and one over; every depth modulo the pipeline
@pytest.mark.parametrize("M,N,K,resid,f32", [
    (1, 32, 128, None, True), (1, 1280, 1280, "f32", True), (31, 96, 256, "bf16", False), (32, 64, 384, None, False),
    (33, 160, 512, "f32", False), (64, 32, 5120, "bf16", True), (65, 32, 128, "f32", True), (127, 96, 256, None, False),
    (129, 288, 384, "bf16", True), (300, 544, 640, "f32", False), (1000, 1280, 1280, "f32", True), (1922, 1280, 5120, "f32", True),
    (2048, 5120, 768, None, False), (8193, 2560, 640, None, False), (5000, 3104, 896, "bf16", True), (30000, 32, 1152, "f32", True)])
def test_linear(M, N, K, resid, f32):
    announce(f"mx4 linear {M}x{N}x{K} resid={resid} f32={f32}")
    r = _rng(M, N, K)
    x, w, b, xh, wh = _operands(r, M, N, K)
    res = r.standard_normal((M, N)).astype(np.float32) if resid else None
    rd = None if resid is None else f32_dev(res) if resid == "f32" else f32_dev(res).bfloat16()
    xq = dn.mx_quantize(dn.DN_MXFP4, f32_dev(x))
    wp = dn.pack_weight(dn.DN_MXFP4, f32_dev(w), N, K)
    want = _matmul(xh, wh) + b
    size = _matmul(np.abs(xh), np.abs(wh)) + np.abs(b)
    if resid:
        want = want + host(rd)
        size = size + np.abs(host(rd))
    tol = (K + 2) * U * size + (0 if f32 else 2.0 ** -8 * np.abs(want))
    for off in (0, 1):  # an output and a residual that are aligned to their elements only
        y = torch.full((M * N + off + 8,), 5.0, device=DEV, dtype=torch.float32 if f32 else torch.bfloat16)
        rr = rd
        if rd is not None and off:
            rr = torch.empty(M * N + 1, device=DEV, dtype=rd.dtype)[1:].view(M, N).copy_(rd)
        dn.op_linear(dn.DN_MXFP4, xq, wp, f32_dev(b), y[off:], M, N, K, resid=rr, resid_f32=resid == "f32", y_f32=f32)
        got = host(y)
        assert (got[:off] == 5.0).all() and (got[off + M * N:] == 5.0).all()
        assert (np.abs(got[off:off + M * N].reshape(M, N) - want) <= tol).all()


# the tile shapes that few tiles per CU, an even number of them and many of them choose, at depths of less than
# their pipelines and of more than the scales that a tile holds at once; the kernel of few rows at that depth
@pytest.mark.parametrize("M,N,K,resid,f32", [
    (2999, 2560, 8320, "bf16", False), (2047, 1248, 8320, "f32", True), (400, 1312, 8576, "bf16", True),
    (2999, 2560, 128, None, True), (2047, 1248, 256, "bf16", False), (900, 1312, 384, "f32", False), (40, 96, 16768, "f32", True)])
def test_linear_tiles(M, N, K, resid, f32):
    test_linear(M, N, K, resid, f32)


@pytest.mark.parametrize("M,N,K,bias", [(2048, 5120, 128, True), (1990, 5056, 384, True), (8100, 1280, 256, False), (600, 2880, 256, True), (580, 2848, 8320, False), (1999, 2560, 8320, True), (1100, 5120, 128, True),
                                        (40, 96, 8576, True)])
def test_linear_geglu_tiles(M, N, K, bias):
    test_linear_geglu(M, N, K, bias)


def test_linear_residual_in_place():
    """y may be the residual's own memory: each value is read before it is written, by the same lanes."""
    for M, N, K in ((5, 64, 128), (700, 1280, 256), (4096, 2560, 256)):
        announce(f"mx4 linear in place {M}x{N}x{K}")
        r = _rng(M, N, K, 5)
        x, w, b, xh, wh = _operands(r, M, N, K)
        xq, wp = dn.mx_quantize(dn.DN_MXFP4, f32_dev(x)), dn.pack_weight(dn.DN_MXFP4, f32_dev(w), N, K)
        y = f32_dev(r.standard_normal((M, N)).astype(np.float32))
        want = torch.empty_like(y)
        dn.op_linear(dn.DN_MXFP4, xq, wp, f32_dev(b), want, M, N, K, resid=y, resid_f32=True, y_f32=True)
        dn.op_linear(dn.DN_MXFP4, xq, wp, f32_dev(b), y, M, N, K, resid=y, resid_f32=True, y_f32=True)
        assert torch.equal(y, want)


def _check_mx(got_buf, y, delta, M, N):
    """An MX4 buffer against exact values y known to within delta: the block's scale is that of a
    largest magnitude within delta, and every value as near as the nearest code of that scale."""
    c, s = mx.from_buffer(got_buf, mx.MXFP4, M, N)
    yb, db = y.reshape(M, -1, 32), np.broadcast_to(delta, y.shape).reshape(M, -1, 32)
    lo = mx.scales((np.sign(yb) * np.maximum(np.abs(yb) - db, 0)).reshape(M, -1), mx.MXFP4)
    hi = mx.scales((np.sign(yb) * (np.abs(yb) + db)).reshape(M, -1), mx.MXFP4)
    assert ((s >= lo) & (s <= hi)).all()
    k = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=1)
    best = np.abs(mx.E2M1[mx.nearest(np.abs(y) / k, mx.MXFP4)] * k - np.abs(y))
    assert (np.abs(mx.values(c, s, mx.MXFP4, N) - y) <= best + 2 * delta).all()


@pytest.mark.parametrize("M,N,K,bias", [(1, 32, 128, True), (33, 96, 256, False), (64, 160, 1280, True), (65, 32, 384, True),
                                        (300, 288, 128, True), (2048, 5120, 1280, True), (1922, 5120, 1280, True), (8192, 2560, 640, True)])
def test_linear_geglu(M, N, K, bias):
    announce(f"mx4 GEGLU {M}x{N}x{K}")
    x, w, b, xh, wh = _operands(_rng(M, N, K, 1), M, 2 * N, K)
    if not bias:
        b[:] = 0
    xq = dn.mx_quantize(dn.DN_MXFP4, f32_dev(x))
    wp = dn.pack_weight(dn.DN_MXFP4, f32_dev(_interleave(w)), 2 * N, K)
    bd = f32_dev(_interleave(b[:, None])[:, 0]) if bias else None
    u = _matmul(xh, wh) + b
    e = (K + 2) * U * (_matmul(np.abs(xh), np.abs(wh)) + np.abs(b))
    a, g, ea, eg = u[:, :N], u[:, N:], e[:, :N], e[:, N:]
    gelu = torch.nn.functional.gelu(torch.from_numpy(g)).numpy()
    want = a * gelu
    tol = ea * np.abs(gelu) + (np.abs(a) + ea) * (1.13 * eg + 4e-7 * np.abs(g)) + 4 * U * np.abs(want)
    y = torch.full((M * N + 4,), 5.0, device=DEV)
    dn.op_linear(dn.DN_MXFP4, xq, wp, bd, y, M, N, K, geglu=True, y_f32=True)
    got = host(y)
    assert (got[M * N:] == 5.0).all() and (np.abs(got[:M * N].reshape(M, N) - want) <= tol).all()
    q = _u8(dn.mx_bytes(dn.DN_MXFP4, M, N))
    dn.op_linear(dn.DN_MXFP4, xq, wp, bd, q, M, N, K, geglu=True)
    q = q.cpu().numpy()
    used = M * (N // 2 + N // 32)
    assert (q[used:] == 0xAA).all()
    _check_mx(q, want, tol, M, N)


@pytest.mark.parametrize("M", [1, 200])
def test_linear_nan_block_stays_in_its_row(M):
    announce(f"mx4 linear, NaN and infinity in a row, M={M}")
    N, K = 96, 256
    x, w, b, xh, wh = _operands(_rng(9), M + 1, N, K)
    x[M // 2, 40] = np.inf
    y = torch.empty(M + 1, N, device=DEV)
    dn.op_linear(dn.DN_MXFP4, dn.mx_quantize(dn.DN_MXFP4, f32_dev(x)), dn.pack_weight(dn.DN_MXFP4, f32_dev(w), N, K), f32_dev(b), y,
                 M + 1, N, K, y_f32=True)
    nan = np.isnan(host(y))
    assert nan[M // 2].all() and nan.sum() == N


def test_linear_operands_past_32_bits():
    """Rows of x and of the output past 2^31 bytes."""
    M, N, K = 2_300_000, 512, 2048
    announce(f"mx4 linear {M}x{N}x{K}: x {M * K // 2 >> 20} MB, y {M * N * 2 >> 20} MB")
    r = _rng(4)
    x, w, b, xh, wh = _operands(r, 64, N, K)
    xq = torch.zeros(dn.mx_bytes(dn.DN_MXFP4, M, K), device=DEV, dtype=torch.uint8)
    c, s = mx.quantize(x, mx.MXFP4)
    part = mx.to_buffer(c, s, mx.MXFP4)
    nc = 64 * K // 2
    xq[M * K // 2 - nc:M * K // 2] = torch.from_numpy(part[:nc]).to(DEV)
    end = M * K // 2 + M * K // 32
    xq[end - 64 * K // 32:end] = torch.from_numpy(part[nc:]).to(DEV)
    y = torch.empty(M, N, device=DEV, dtype=torch.bfloat16)
    dn.op_linear(dn.DN_MXFP4, xq, dn.pack_weight(dn.DN_MXFP4, f32_dev(w), N, K), f32_dev(b), y, M, N, K)
    want = _matmul(xh, wh) + b
    tol = (K + 2) * U * (_matmul(np.abs(xh), np.abs(wh)) + np.abs(b)) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(host(y[-64:]) - want) <= tol).all()
    assert torch.equal(y[:-64], f32_dev(b).bfloat16().expand(M - 64, N))
    del xq, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,C", [(1, 32), (5, 96), (300, 1280), (2048, 640), (3, 2048)])
def test_layernorm(M, C):
    """Exact values are known to within the fp32 statistics: mean, variance and two products, a few
    units of the normalised value (10) and of the shift."""
    announce(f"mx4 layernorm {M}x{C}")
    r = _rng(M, C)
    x = (1.0 + 3.0 * r.standard_normal((M, C))).astype(np.float32)
    g = (1 + 0.1 * r.standard_normal(C)).astype(np.float32)
    b = (0.1 * r.standard_normal(C)).astype(np.float32)
    q = _u8(dn.mx_bytes(dn.DN_MXFP4, M, C))
    dn.op_layernorm(dn.DN_MXFP4, f32_dev(x), q, M, C, f32_dev(g), f32_dev(b), 1e-5)
    ref = L.layer_norm(x.astype(np.float64), g.astype(np.float64), b.astype(np.float64), 1e-5)
    q = q.cpu().numpy()
    assert (q[M * (C // 2 + C // 32):] == 0xAA).all()
    _check_mx(q, ref, 40 * U * (np.abs(ref) + np.abs(b) + 1.0), M, C)


# ----------------------------------------------------------------------------- the search

def _search(fmt, x, q, tab=None, stream=None):
    n, dim = x.shape
    nq = q.shape[0]
    table = dn.mx_quantize(fmt, torch.from_numpy(x).to(DEV))
    idx = torch.full((nq,), -9, device=DEV, dtype=torch.int64)
    score = torch.full((nq,), float("nan"), device=DEV)
    k = torch.full((nq,), -9, device=DEV, dtype=torch.int32) if tab else None
    ws = _u8(dn.ac_mx_lookup_bytes(nq, n, dim), 0xFF)
    dn.ac_mx_lookup(fmt, torch.from_numpy(q).to(DEV), table, n, ws, idx, score, k, *(tab or (None, None)))
    return idx.cpu().numpy(), score.cpu().numpy(), k.cpu().numpy() if tab else None


def _cosines(fmt, x, q):
    v = mx.rounded(x, fmt)
    v = v * 2.0 ** -np.floor(np.log2(np.maximum(np.abs(v).max(1, keepdims=True), 1e-300)))
    with np.errstate(invalid="ignore", divide="ignore"):
        c = _matmul(q.astype(np.float64) / np.linalg.norm(q.astype(np.float64), axis=1, keepdims=True),
                    v / np.linalg.norm(v, axis=1, keepdims=True))
    return np.where(np.isnan(c), -np.inf, c)


def _planted(r, n, dim, nq):
    x = r.standard_normal((n, dim)).astype(np.float32)
    rows = r.integers(0, n, nq)
    q = x[rows] + 0.3 * r.standard_normal((nq, dim))
    return x, (q / np.linalg.norm(q, axis=1, keepdims=True)).astype(np.float16)


def _check_search(fmt, x, q, got):
    """The row of a cosine within the sums' rounding of the largest (each a sum of dim exact products:
    2 dim 2^-24, and a few units for the norms), and its cosine."""
    idx, score, _ = got
    c = _cosines(fmt, x, q)
    tol = (2 * x.shape[1] + 16) * U
    best = c.max(1)
    assert ((idx >= 0) & (idx < x.shape[0])).all()
    at = c[np.arange(len(idx)), idx]
    assert (at >= best - tol).all()
    assert (np.abs(score - at) <= tol).all()
    clear = np.sort(c, 1)[:, -2] < best - 2 * tol if x.shape[0] > 1 else np.ones(len(idx), bool)
    assert np.array_equal(idx[clear], c.argmax(1)[clear])


@pytest.mark.parametrize("n,dim,nq", [(1, 1, 1), (1, 40, 7), (2, 31, 2), (31, 32, 3), (33, 33, 5), (63, 64, 32), (65, 100, 33),
                                      (300, 256, 4), (1000, 250, 64), (4097, 500, 9), (4097, 512, 70), (2000, 768, 1), (2000, 768, 130),
                                      (700, 1000, 40), (700, 1024, 3), (700, 1024, 64), (500, 1025, 6), (200, 9000, 3), (50, 16384, 2),
                                      (70001, 768, 2), (70001, 768, 64), (100000, 256, 6)])
@pytest.mark.parametrize("fmt", FMTS)
def test_lookup(fmt, n, dim, nq):
    announce(f"mx lookup fmt={fmt} n={n} dim={dim} nq={nq}")
    x, q = _planted(_rng(n, dim, nq), n, dim, nq)
    _check_search(fmt, x, q, _search(fmt, x, q))


# row lengths around those that change kernel or registers, odd ones whose queries begin at any address; query
# counts around the groups of 16
@pytest.mark.parametrize("dim", [7, 8, 9, 33, 255, 257, 512, 513, 768, 769, 1023, 1024, 1025])
@pytest.mark.parametrize("fmt", FMTS)
def test_lookup_lengths_and_groups(fmt, dim):
    for n, nq in ((1, 1), (17, 16), (1000, 17), (1030, 32), (700, 33), (1500, 64), (300, 70)):
        test_lookup(fmt, n, dim, nq)


@pytest.mark.parametrize("nq", [1, 2, 40])
@pytest.mark.parametrize("dim", [96, 768, 1056])
@pytest.mark.parametrize("fmt", FMTS)
def test_lookup_scales_of_any_size(fmt, dim, nq):
    """Rows 2^-90 to 2^90 times as large, blocks of a row 2^-12 to 2^12: cosines do not see the first and
    must not lose the second."""
    announce(f"mx lookup, wide scales fmt={fmt} dim={dim} nq={nq}")
    r = _rng(dim, nq, 5)
    x, q = _planted(r, 500, dim, nq)
    f = (2.0 ** r.integers(-12, 13, (1, dim // 32))).repeat(32, 1)
    x = (x * f * 2.0 ** r.integers(-90, 91, (500, 1))).astype(np.float32)
    q = (q.astype(np.float32) / np.abs(f)).astype(np.float16)
    _check_search(fmt, x, q, _search(fmt, x, q))


@pytest.mark.parametrize("scale", [2.0 ** -22, 2.0 ** -14, 2.0 ** 12])
@pytest.mark.parametrize("dim", [5, 64, 768, 1100])
@pytest.mark.parametrize("fmt", FMTS)
def test_lookup_queries_of_any_size(fmt, dim, scale):
    """Queries of fp16 values below its normal range and near its largest: cosines of what they hold."""
    announce(f"mx lookup, queries of size {scale} fmt={fmt} dim={dim}")
    for nq in (1, 20):
        x, q = _planted(_rng(dim, nq, 6), 300, dim, nq)
        q = (q.astype(np.float64) * scale).astype(np.float16)
        q[0, 0] = np.float16(scale)
        idx, score, _ = _search(fmt, x, q)
        # a component of a unit vector below 2^-3 is below half of fp16's least, 2^-24, when scaled by 2^-22, hence
        # some queries hold zeros only, and a zero query finds nothing
        on = (q != 0).any(1)
        assert on[0] and (idx[~on] == -1).all() and (score[~on] == 0).all()
        _check_search(fmt, x, q[on], (idx[on], score[on], None))


@pytest.mark.parametrize("n,nq", [(200, 1), (200, 3), (200, 64), (5000, 2), (5000, 33)])
@pytest.mark.parametrize("dim", [64, 768, 1100])
@pytest.mark.parametrize("fmt", FMTS)
def test_lookup_ties_zero_and_nan(fmt, dim, n, nq):
    announce(f"mx lookup ties, zeros, NaN fmt={fmt} dim={dim} n={n} nq={nq}")
    r = _rng(dim, n, nq)
    x = r.standard_normal((n, dim)).astype(np.float32)
    x[3] = 0
    x[7, dim // 2] = np.nan
    x[n - 2] = x[n // 2] = x[11]      # the same row three times: the lowest index
    x[n - 1] = 4 * x[12]              # a multiple of a row: the same cosine
    q = np.stack([x[11], x[12], x[7], x[3]]).astype(np.float16)[np.arange(nq) % 4]
    q[np.isnan(q)] = 1.0
    idx, score, k = _search(fmt, x, q, ([0.5, 0.9], [4, 8, 16]))
    for j in range(nq):
        if j % 4 < 2:
            assert idx[j] == 11 + j % 4 and score[j] > 0.95 and k[j] == 16
        elif j % 4 == 2:
            assert idx[j] not in (3, 7) and idx[j] >= 0
        else:
            assert (idx[j], score[j], k[j]) == (-1, 0.0, 0)


@pytest.mark.parametrize("nq", [1, 5])
def test_lookup_nothing_to_find(nq):
    announce(f"mx lookup: zero table, NaN table, queries that are not finite, nq={nq}")
    for x in (np.zeros((40, 96), np.float32), np.full((40, 96), np.nan, np.float32)):
        idx, score, k = _search(dn.DN_MXFP4, x, np.ones((nq, 96), np.float16), ([0.0], [3, 5]))
        assert (idx == -1).all() and (score == 0).all() and (k == 0).all()
    q = np.ones((nq, 96), np.float16)
    q[0, 5] = np.inf
    q[-1, 7] = np.nan
    idx, score, _ = _search(dn.DN_MXFP8, np.ones((40, 96), np.float32), q)
    assert idx[0] == -1 and idx[-1] == -1 and score[0] == score[-1] == 0
    assert (idx[1:-1] == 0).all()


def test_lookup_levels_are_those_of_the_reported_cosine():
    announce("mx lookup levels")
    x, q = _planted(_rng(8), 3000, 256, 64)
    thr = [0.2, 0.5, 0.94, 0.955, 0.96]
    idx, score, k = _search(dn.DN_MXFP4, x, q, (thr, [0, 5, 10, 15, 20, 25]))
    assert np.array_equal(k, np.array([0, 5, 10, 15, 20, 25])[(score[:, None] >= np.float32(thr)).sum(1)])


# ----------------------------------------------------------------------------- together

def test_calls_without_a_stream_take_the_current_one():
    announce("current stream")
    side = torch.cuda.Stream()
    for _ in range(2):
        assert dn._stream(None) == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(side):
            assert dn._stream(None) == side.cuda_stream == dn._stream(side)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                assert dn._stream(None) == torch.cuda.current_stream().cuda_stream != side.cuda_stream
                torch.zeros(1, device=DEV)


def test_streams_and_graphs():
    """Store, search, fetch and the feed-forward on a side stream and captured into two graphs with
    workspaces of their own, replayed in turn: every result equals the eager one bit for bit."""
    announce("mx operators on a side stream and in graphs")
    r = _rng(12)
    n, dim, M, C = 3000, 256, 300, 128
    emb = torch.from_numpy(r.standard_normal((n, dim)).astype(np.float16)).to(DEV)
    q = (emb[[5, 77, 2999, 1500, 8]] + 0.1).contiguous()
    x = f32_dev(r.standard_normal((M, C)))
    g, b = f32_dev(1 + 0.1 * r.standard_normal(C)), f32_dev(0.1 * r.standard_normal(C))
    w1 = dn.pack_weight(dn.DN_MXFP4, f32_dev(_interleave(r.standard_normal((8 * C, C)) / 11)), 8 * C, C)
    w2 = dn.pack_weight(dn.DN_MXFP4, f32_dev(r.standard_normal((C, 4 * C)) / 22), C, 4 * C)
    slots = torch.from_numpy(r.permutation(n)).to(DEV)

    def buffers():
        return dict(table=_u8(dn.mx_bytes(dn.DN_MXFP8, n, dim), 0), ws=_u8(dn.ac_mx_store_bytes(n, n)),
                    lws=_u8(dn.ac_mx_lookup_bytes(5, n, dim)), idx=torch.full((5,), -5, device=DEV), score=torch.zeros(5, device=DEV),
                    out=torch.zeros(5, dim, device=DEV), a=_u8(dn.mx_bytes(dn.DN_MXFP4, M, C)), h=_u8(dn.mx_bytes(dn.DN_MXFP4, M, 4 * C)),
                    y=torch.zeros(M, C, device=DEV))

    def run(d, stream):
        dn.ac_mx_store(dn.DN_MXFP8, emb, slots, d["table"], n, d["ws"], stream=stream)
        dn.ac_mx_lookup(dn.DN_MXFP8, q, d["table"], n, d["lws"], d["idx"], d["score"], stream=stream)
        dn.ac_mx_fetch(dn.DN_MXFP8, d["table"], n, d["idx"], d["out"], stream=stream)
        dn.op_layernorm(dn.DN_MXFP4, x, d["a"], M, C, g, b, 1e-5, stream=stream)
        dn.op_linear(dn.DN_MXFP4, d["a"], w1, None, d["h"], M, 4 * C, C, geglu=True, stream=stream)
        dn.op_linear(dn.DN_MXFP4, d["h"], w2, None, d["y"], M, C, 4 * C, resid=x, resid_f32=True, y_f32=True, stream=stream)

    eager = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(eager, side)
    side.synchronize()
    assert eager["idx"].tolist() == slots[[5, 77, 2999, 1500, 8]].tolist()
    sets = [buffers(), buffers()]
    torch.cuda.synchronize()
    graphs = []
    for d in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            run(d, torch.cuda.current_stream())
        graphs.append(gr)
    for rep in range(4):
        for d in sets:
            for k in ("idx", "score", "out", "y"):
                d[k].fill_(-5)
        again = buffers()
        if rep % 2:
            run(again, torch.cuda.current_stream())
            torch.cuda.synchronize()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for d in sets + ([again] if rep % 2 else []):
            for k in ("table", "idx", "score", "out", "a", "h", "y"):
                u = (d[k], eager[k]) if k not in ("a", "h") else (d[k][:-16], eager[k][:-16])
                assert torch.equal(*u), (rep, k)


def test_a_prompt_resumes_from_the_quantized_cache():
    """As a worker uses them: the states of a run are captured and stored in 8 bits with the prompt's
    embedding, a similar prompt finds them, fetches the state of its level and runs the rest."""
    announce("capture -> store -> lookup -> fetch -> resume (tiny denoiser)")
    cfg = W.tiny(W.DN_BF16)
    model = dn.Denoiser(cfg, W.weight_blob(dn.weight_table(cfg), 42))
    ts, ctx = S.default_timesteps(10), f32_dev(W.text_ctx(cfg))
    caps = [2, 4, 6]
    states = torch.empty(3, 1, 4, 16, 16, device=DEV, dtype=torch.bfloat16)
    model.denoise_capture(f32_dev(W.latent(cfg, 0)), ctx, ts, 0, 10, 7.5, caps, states)
    n, dim, numel = 50, 768, 4 * 16 * 16
    emb = torch.from_numpy(W.cache_embeddings(n, dim)).to(DEV)
    fmt = dn.DN_MXFP8
    etab = dn.mx_quantize(fmt, emb)
    ltab = torch.zeros(dn.mx_bytes(fmt, 3 * n, numel), device=DEV, dtype=torch.uint8)
    mine = 17
    dn.ac_mx_store(fmt, states.view(3, numel), torch.arange(3, device=DEV) + 3 * mine, ltab, 3 * n)
    noise = torch.from_numpy(W.normal((1, dim), 3)).to(DEV) / dim ** 0.5
    q = (0.9 * emb[mine:mine + 1].float() + 0.35 * noise).half()
    idx, score, k = (torch.empty(1, device=DEV, dtype=t) for t in (torch.int64, torch.float32, torch.int32))
    dn.ac_mx_lookup(fmt, q, etab, n, _u8(dn.ac_mx_lookup_bytes(1, n, dim)), idx, score, k, [0.5, 0.8, 0.95], [0, 2, 4, 6])
    assert idx.item() == mine and k.item() == 4
    lat = torch.empty(1, numel, device=DEV)
    dn.ac_mx_fetch(fmt, ltab, 3 * n, 3 * idx + caps.index(k.item()), lat)
    assert np.array_equal(host(lat), mx.rounded(host(states[1].view(1, numel)), mx.MXFP8))
    a, b = lat.view(1, 4, 16, 16).clone(), states[1].float()
    model.denoise(a, ctx, ts, 4, 6, 7.5)
    model.denoise(b, ctx, ts, 4, 6, 7.5)
    torch.cuda.synchronize()
    announce(f"  final latent from the 8-bit state against the bf16 state: rel-L2 {rel_l2(host(a), host(b)):.3e}")
    assert torch.isfinite(a).all() and not torch.equal(a, b)
    model.close()


def test_tiny_denoiser_with_a_4_bit_feed_forward(monkeypatch):
    """The DN_MXFP4 model against the oracle emulating its quantisation. As for the fp8 variant at depth,
    the bar is the oracle's own displacement when it rounds its activations to bf16 as the library
    stores them: a rounding boundary turns a small difference into a whole step of the format.
    Both displacements are draws of one size, hence the factor 1.5."""
    from tests.test_gpu_denoise import _bf16_activations
    announce("tiny mx4 feed-forward variant: steps vs oracle")
    cfg = W.tiny(W.DN_MXFP4).with_(model_channels=128, levels=((128, 1, 4, 32),))
    blob = W.weight_blob(dn.weight_table(cfg), 42)
    model, bf16 = dn.Denoiser(cfg, blob), dn.Denoiser(cfg.with_(dtype=W.DN_BF16), blob)
    Wt = mx.mx4_model_weights(unet.unpack(cfg, blob))
    x, ctx = W.latent(cfg, 0), W.text_ctx(cfg)

    def eps(m):
        raw = torch.empty((2, 4, 16, 16), device=DEV)
        m.unet_eps(f32_dev(x), t, f32_dev(ctx), 7.5, raw)
        torch.cuda.synchronize()
        return raw.cpu().numpy()

    for t, tp in ((901, 801), (1, -1)):
        ref, _, _ = sampler.step(cfg, Wt, x, ctx, t, tp, 7.5, ff_act=mx.mx4_act)
        with monkeypatch.context() as mp:
            _bf16_activations(mp)
            ref_b, _, _ = sampler.step(cfg, Wt, x, ctx, t, tp, 7.5, ff_act=mx.mx4_act)
        e, spread, effect = rel_l2(eps(model), ref), rel_l2(ref_b, ref), rel_l2(eps(model), eps(bf16))
        announce(f"  t={t}: rel-L2 vs the oracle {e:.3e}, its displacement {spread:.3e}, effect of the 4 bits {effect:.3e}")
        assert e <= max(2e-2, 1.5 * spread)
        assert effect > e
    model.close()
    bf16.close()
