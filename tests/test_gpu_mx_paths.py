"""Paths of the microscaled operators that whole models take and single calls of few rows do not:
tiles of every shape with NaN and infinite blocks, the LayerNorm that completes a split product,
the residual stream in place, captured feed-forwards of tile size, denoisers with DN_MXFP4.

Tolerances are those of test_gpu_mx."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layers as L, mx, sampler, schedule as S, unet
from paper_2511_06724_amd import dn, workloads as W
from tests.gpu_util import DEV, announce, f32_dev, host, rel_l2
from tests.plans import LINEAR, plan
from tests.test_gpu_mx import U, _check_mx, _interleave, _operands, _rng, _u8
from tests.test_mx_plans_cpu import plan as plan_mx4

pytestmark = pytest.mark.gpu

F4 = dn.DN_MXFP4
ROWS, SMALL, FIVE, BIG = (32, 32), (64, 128), (64, 160), (128, 256)
# (M, output columns, K) per GEGLU kernel: few rows, tiles of 64 rows, of 128 rows, and both in one launch
GEGLU = [((40, 96, 256), (32, 64, 0)), ((300, 2560, 256), (128, 256, 20)), ((4200, 1280, 256), (128, 256, 0)), ((2048, 5120, 256), (128, 256, 8))]


def _nan_blocks(q, M, N):
    """Blocks of an MX4 buffer that are NaN, [M, N / 32]; their codes must be zero."""
    c, s = mx.from_buffer(q.cpu().numpy(), mx.MXFP4, M, N)
    nan = s == 255
    assert (c.reshape(M, -1, 32)[nan] == 0).all()
    return nan


def test_dequantize_allocates_fp32_whatever_the_default_type():
    announce("mx_dequantize under another default type")
    x = torch.randn(5, 70, device=DEV)
    q = dn.mx_quantize(dn.DN_MXFP8, x)
    want = dn.mx_dequantize(dn.DN_MXFP8, q, 5, 70)
    torch.set_default_dtype(torch.float64)
    try:
        got = dn.mx_dequantize(dn.DN_MXFP8, q, 5, 70)
    finally:
        torch.set_default_dtype(torch.float32)
    assert got.dtype is torch.float32 and torch.equal(got, want)


# ----------------------------------------------------------------------------- NaN and infinities

@pytest.mark.parametrize("shape,tile", [((201, 96, 256), ROWS), ((700, 1280, 256), SMALL), ((2048, 1280, 256), FIVE), ((2000, 1248, 896), FIVE),
                                        ((8000, 672, 2560), BIG), ((400, 1312, 8576), SMALL)])
def test_linear_nan_blocks(shape, tile):
    """A row of x with an infinity is NaN everywhere, a row of w with a NaN is a column of NaN, and nothing else changes."""
    M, N, K = shape
    announce(f"mx4 linear, NaN blocks {shape} {plan_mx4(M, N, K)}")
    assert plan_mx4(M, N, K)[:2] == tile
    x, w, b, _, _ = _operands(_rng(M, N, 31), M, N, K)
    bd, y = f32_dev(b), torch.empty(2, M, N, device=DEV)
    for i in range(2):
        if i:
            x[M // 2, K - 30], x[M - 1, 5], w[N // 3, 40] = np.inf, np.nan, -np.inf
        dn.op_linear(F4, dn.mx_quantize(F4, f32_dev(x)), dn.pack_weight(F4, f32_dev(w), N, K), bd, y[i], M, N, K, y_f32=True)
    want = torch.zeros(M, N, device=DEV, dtype=torch.bool)
    want[M // 2] = want[M - 1] = True
    want[:, N // 3] = True
    assert torch.equal(torch.isnan(y[1]), want)
    assert torch.equal(y[0][~want], y[1][~want])


@pytest.mark.parametrize("shape,tile", GEGLU)
def test_geglu_nan_blocks(shape, tile):
    """A NaN of a row or of a weight column makes exactly the blocks it enters NaN blocks; a gate of +-infinity
    (an infinite bias) gives an infinite or a zero value: the infinite one makes its block NaN as well."""
    M, N, K = shape
    announce(f"mx4 GEGLU, NaN blocks {shape}")
    assert plan_mx4(M, 2 * N, K, True) == tile
    x, w, b, _, _ = _operands(_rng(M, N, 32), M, 2 * N, K)
    q = [_u8(dn.mx_bytes(F4, M, N)) for _ in range(2)]
    for i in range(2):
        if i:
            x[M // 2, K - 30], x[M - 1, 5] = np.inf, np.nan
            w[N - 1, 40] = np.nan            # value column N - 1
            w[N + 33, 7] = np.inf            # gate column 33
            b[N], b[N + 70] = -np.inf, np.inf  # gates of columns 0 (its values become -0 or 0) and 70
        dn.op_linear(F4, dn.mx_quantize(F4, f32_dev(x)), dn.pack_weight(F4, f32_dev(_interleave(w)), 2 * N, K),
                     f32_dev(_interleave(b[:, None])[:, 0]), q[i], M, N, K, geglu=True)
    assert not _nan_blocks(q[0], M, N).any()
    got = _nan_blocks(q[1], M, N)
    want = np.zeros((M, N // 32), bool)
    want[[M // 2, M - 1]] = True
    want[:, [1, 2, N // 32 - 1]] = True
    assert np.array_equal(got, want)
    # column 0 is zero in the other rows; every other block is what it was
    (c0, s0), (c1, s1) = (mx.from_buffer(t.cpu().numpy(), mx.MXFP4, M, N) for t in q)
    rest = ~want
    rest[:, 0] = False
    assert np.array_equal(s0[rest], s1[rest]) and np.array_equal(c0.reshape(M, -1, 32)[rest], c1.reshape(M, -1, 32)[rest])
    rows = np.setdiff1d(np.arange(M), [M // 2, M - 1])
    assert (c1[rows, 0] % 8 == 0).all()


def test_layernorm_nan_blocks():
    announce("mx4 layernorm, NaN rows and an infinite scale")
    M, Cc = 300, 640
    r = _rng(33)
    x, g, b = r.standard_normal((M, Cc)).astype(np.float32), np.ones(Cc, np.float32), np.zeros(Cc, np.float32)
    g[100] = np.inf
    x[7, 639], x[299, 0] = np.inf, np.nan
    q = _u8(dn.mx_bytes(F4, M, Cc))
    dn.op_layernorm(F4, f32_dev(x), q, M, Cc, f32_dev(g), f32_dev(b), 1e-5)
    want = np.zeros((M, Cc // 32), bool)
    want[[7, 299]] = True
    want[:, 3] = True
    assert np.array_equal(_nan_blocks(q, M, Cc), want)


# ----------------------------------------------------------------------------- the residual stream

@pytest.mark.parametrize("M,Cc,nsplit,bias,resid", [(512, 1280, 3, True, True), (301, 320, 1, False, True), (77, 2048, 8, True, True),
                                                    (5, 32, 2, True, False), (1030, 640, 4, False, False), (64, 96, 5, True, True),
                                                    (33, 1280, 6, True, True), (130, 128, 7, False, True)])
def test_layernorm_of_partial_slabs(M, Cc, nsplit, bias, resid):
    """The LayerNorm that sums a split product's slabs into the residual stream, with an MX4 output (the
    attention's out-projection before the feed-forward): no entry point but the denoiser's reaches it."""
    announce(f"mx4 layernorm of {nsplit} slabs {M}x{Cc} bias={bias} resid={resid}")
    f = getattr(dn.lib, "_ZN2dn16layernorm_reduceINS_6Mx4RowEEEvPfPT_xiPKfS6_fS6_iS6_bP12ihipStream_t")
    P = C.c_void_p
    f.argtypes, f.restype = [P, P, C.c_longlong, C.c_int, P, P, C.c_float, P, C.c_int, P, C.c_bool, P], None
    r = _rng(M, Cc, nsplit)
    x = (0.5 + 2.0 * r.standard_normal((M, Cc))).astype(np.float32)
    slabs = r.standard_normal((nsplit, M, Cc)).astype(np.float32)
    bv = r.standard_normal(Cc).astype(np.float32)
    g, b = (1 + 0.1 * r.standard_normal(Cc)).astype(np.float32), (0.1 * r.standard_normal(Cc)).astype(np.float32)
    xd, sd, bd, gd, ld, q = f32_dev(x), f32_dev(slabs), f32_dev(bv), f32_dev(g), f32_dev(b), _u8(dn.mx_bytes(F4, M, Cc))
    f(xd.data_ptr(), q.data_ptr(), M, Cc, gd.data_ptr(), ld.data_ptr(), 1e-5, sd.data_ptr(), nsplit, bd.data_ptr() if bias else None, resid,
      torch.cuda.current_stream().cuda_stream)
    terms = [x.astype(np.float64)] * resid + [np.broadcast_to(bv.astype(np.float64), x.shape)] * bias + list(slabs.astype(np.float64))
    got = host(xd)
    assert (np.abs(got - sum(terms)) <= len(terms) * U * sum(np.abs(t) for t in terms)).all()
    # the values normalised are those written back
    ref = L.layer_norm(got, g.astype(np.float64), b.astype(np.float64), 1e-5)
    q = q.cpu().numpy()
    assert (q[M * (Cc // 2 + Cc // 32):] == 0xAA).all()
    _check_mx(q, ref, 40 * U * (np.abs(ref) + np.abs(b) + 1.0), M, Cc)


@pytest.mark.parametrize("M,N,K,off", [(5, 64, 128, 0), (700, 1280, 256, 0), (2000, 1248, 896, 0), (8000, 672, 2560, 0), (4100, 2592, 128, 1)])
def test_linear_bf16_residual_in_place(M, N, K, off):
    announce(f"mx4 linear, bf16 in place {M}x{N}x{K} offset {off}")
    r = _rng(M, N, K, 6)
    x, w, b, _, _ = _operands(r, M, N, K)
    xq, wp = dn.mx_quantize(F4, f32_dev(x)), dn.pack_weight(F4, f32_dev(w), N, K)
    y = torch.empty(M * N + 8, device=DEV, dtype=torch.bfloat16)[off:off + M * N].view(M, N).copy_(f32_dev(r.standard_normal((M, N))))
    want = torch.empty_like(y)
    dn.op_linear(F4, xq, wp, f32_dev(b), want, M, N, K, resid=y)
    dn.op_linear(F4, xq, wp, f32_dev(b), y, M, N, K, resid=y)
    assert torch.equal(y, want)


def test_captured_feed_forward_of_tile_size():
    """LayerNorm, GEGLU layer (tiles of 128 and of 64 rows) and output layer in a graph, replayed with eager work
    and changed inputs between: every replay equals the eager pass bit for bit."""
    M, Cc = 2048, 1280
    announce(f"mx4 feed-forward {M}x{Cc} in a graph")
    r = _rng(34)
    g, b = f32_dev(1 + 0.1 * r.standard_normal(Cc)), f32_dev(0.1 * r.standard_normal(Cc))
    w1 = dn.pack_weight(F4, f32_dev(_interleave(r.standard_normal((8 * Cc, Cc)) / Cc ** 0.5)), 8 * Cc, Cc)
    w2 = dn.pack_weight(F4, f32_dev(r.standard_normal((Cc, 4 * Cc)) / (4 * Cc) ** 0.5), Cc, 4 * Cc)
    assert plan_mx4(M, 8 * Cc, Cc, True)[2] > 0 and plan_mx4(M, Cc, 4 * Cc)[0] > 32
    xs = [f32_dev(r.standard_normal((M, Cc))) for _ in range(3)]
    x, a, h, y = xs[0].clone(), _u8(dn.mx_bytes(F4, M, Cc)), _u8(dn.mx_bytes(F4, M, 4 * Cc)), torch.empty(M, Cc, device=DEV)

    def run():
        dn.op_layernorm(F4, x, a, M, Cc, g, b, 1e-5)
        dn.op_linear(F4, a, w1, None, h, M, 4 * Cc, Cc, geglu=True)
        dn.op_linear(F4, h, w2, None, y, M, Cc, 4 * Cc, resid=x, resid_f32=True, y_f32=True)

    want = []
    for v in xs:
        x.copy_(v)
        run()
        want.append((h.clone(), y.clone()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(6):
        x.copy_(xs[rep % 3])
        h.fill_(rep), y.fill_(-5)
        if rep % 2:
            run()
            torch.cuda.synchronize()
            y.fill_(-6)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h[:-16], want[rep % 3][0][:-16]) and torch.equal(y, want[rep % 3][1]), rep


# ----------------------------------------------------------------------------- denoisers

def test_denoiser_of_two_blocks_on_tiles(monkeypatch):
    """A 1280-wide denoiser of two transformer blocks on 16 x 16 latents: both products run as tiles, the first
    block's output layer adds to the fp32 residual stream in place, and the LayerNorm before each feed-forward
    sums the slabs of a split out-projection. Bar as in test_tiny_denoiser_with_a_4_bit_feed_forward."""
    from tests.test_gpu_denoise import _bf16_activations
    announce("1280-wide mx4 feed-forward variant, two blocks: steps vs oracle")
    cfg = W.tiny(W.DN_MXFP4).with_(model_channels=320, levels=((1280, 2, 20, 64),))
    M, Cc = 2 * 16 * 16, 1280
    assert plan_mx4(M, 8 * Cc, Cc, True)[0] == 128 and plan_mx4(M, Cc, 4 * Cc)[0] > 32
    assert plan(M, Cc, Cc, LINEAR, fused_reduce=True, out_f32=True).split > 1
    blob = W.weight_blob(dn.weight_table(cfg), 43)
    model, bf16 = dn.Denoiser(cfg, blob), dn.Denoiser(cfg.with_(dtype=W.DN_BF16), blob)
    Wt = mx.mx4_model_weights(unet.unpack(cfg, blob))
    x, ctx = W.latent(cfg, 0), W.text_ctx(cfg)

    def eps(m):
        raw = torch.empty((2, 4, 16, 16), device=DEV)
        m.unet_eps(f32_dev(x), 901, f32_dev(ctx), 7.5, raw)
        torch.cuda.synchronize()
        return raw.cpu().numpy()

    ref, _, _ = sampler.step(cfg, Wt, x, ctx, 901, 801, 7.5, ff_act=mx.mx4_act)
    announce("  oracle step done")
    with monkeypatch.context() as mp:
        _bf16_activations(mp)
        ref_b, _, _ = sampler.step(cfg, Wt, x, ctx, 901, 801, 7.5, ff_act=mx.mx4_act)
    got, got16 = eps(model), eps(bf16)
    e, spread, effect = rel_l2(got, ref), rel_l2(ref_b, ref), rel_l2(got, got16)
    announce(f"  rel-L2 vs the oracle {e:.3e}, its displacement {spread:.3e}, effect of the 4 bits {effect:.3e}")
    assert e <= max(2e-2, 1.5 * spread)
    assert effect > e
    model.close()
    bf16.close()


@pytest.mark.parametrize("batch", [1, 3])
def test_denoiser_resumes_bitwise(batch):
    """Runs repeat, resume at any iteration and capture their states bit for bit, as the other variants' do."""
    announce(f"mx4 denoiser: determinism, resume, capture, batch {batch}")
    cfg = W.tiny(W.DN_MXFP4).with_(model_channels=128, levels=((128, 2, 4, 32),), batch=batch)
    model = dn.Denoiser(cfg, W.weight_blob(dn.weight_table(cfg), 44))
    x, cd, ts = W.latent(cfg, 0), f32_dev(W.text_ctx(cfg)), S.default_timesteps(10)
    a, b, c = f32_dev(x), f32_dev(x), f32_dev(x)
    model.denoise(a, cd, ts, 0, 10, 7.5)
    model.denoise(b, cd, ts, 0, 4, 7.5)
    mid = b.clone()
    model.denoise(b, cd, ts, 4, 6, 7.5)
    slots = torch.empty((2, *a.shape), device=DEV, dtype=torch.bfloat16)
    model.denoise_capture(c, cd, ts, 0, 10, 7.5, [4, 10], slots)
    torch.cuda.synchronize()
    assert torch.isfinite(a).all() and torch.equal(a, b) and torch.equal(a, c)
    assert torch.equal(slots[0], mid.bfloat16()) and torch.equal(slots[1], a.bfloat16())
    model.close()


def test_sdxl_step_properties_with_a_4_bit_feed_forward():
    """The SD-XL-shaped UNet with DN_MXFP4: finite, repeatable, resumed bit for bit, and further from the bf16
    model than DN_FP8 is (it is the coarser level)."""
    announce("sdxl mx4 properties")
    g = torch.Generator(device=DEV).manual_seed(12)
    x, ctx = torch.randn((1, 4, 128, 128), device=DEV, generator=g), torch.randn((2, 77, 2048), device=DEV, generator=g)
    ts = S.default_timesteps(50)
    blob = W.weight_blob_device(dn.weight_table(W.sdxl()), 11, DEV)
    raw = {}
    for dt in (W.DN_BF16, W.DN_FP8, W.DN_MXFP4):
        model = dn.Denoiser(W.sdxl(dt), blob)
        raw[dt] = torch.empty((2, 4, 128, 128), device=DEV)
        model.unet_eps(x, 981, ctx, 7.5, raw[dt])
        if dt == W.DN_MXFP4:
            a, b = x.clone(), x.clone()
            model.denoise(a, ctx, ts, 0, 3, 7.5)
            model.denoise(b, ctx, ts, 0, 1, 7.5)
            model.denoise(b, ctx, ts, 1, 2, 7.5)
            torch.cuda.synchronize()
            assert torch.isfinite(a).all() and torch.equal(a, b)
        model.close()
    e8, e4 = (rel_l2(host(raw[d]), host(raw[W.DN_BF16])) for d in (W.DN_FP8, W.DN_MXFP4))
    announce(f"  rel-L2 from the bf16 model: fp8 {e8:.3e}, mx4 {e4:.3e}")
    assert e8 < e4
    del blob
    torch.cuda.empty_cache()


# ----------------------------------------------------------------------------- at once, and at the limits

@pytest.mark.parametrize("n,dim", [(200, 33), (4000, 96)])
def test_calls_at_once(n, dim):
    """Two streams store into alternate slots of one table (neighbours' scales share words and lines), then search
    and read it, each with workspaces of its own: as one after the other."""
    announce(f"mx stores, searches and fetches on two streams, {n} x {dim}")
    fmt = dn.DN_MXFP8
    x = f32_dev(_rng(n, dim, 41).standard_normal((n, dim))).half()
    want = dn.mx_quantize(fmt, x)[:n * 33 * (-(-dim // 32))]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(5):
        table = _u8(dn.mx_bytes(fmt, n, dim), rep)
        slots = [torch.arange(i, n, 2, device=DEV) for i in range(2)]
        rows = [x[i::2].contiguous() for i in range(2)]
        ws = [_u8(max(1, dn.ac_mx_store_bytes(len(s), n))) for s in slots]
        lws = [_u8(dn.ac_mx_lookup_bytes(40, n, dim)) for _ in range(2)]
        idx = [torch.full((40,), -5, device=DEV) for _ in range(2)]
        out = [torch.zeros(40, dim, device=DEV) for _ in range(2)]
        q = [x[i:i + 80:2].contiguous() for i in range(2)]
        torch.cuda.synchronize()
        for i, st in enumerate(streams):
            dn.ac_mx_store(fmt, rows[i], slots[i], table, n, ws[i], stream=st)
        torch.cuda.synchronize()
        assert torch.equal(table[:want.numel()], want), rep
        for i, st in enumerate(streams):
            dn.ac_mx_lookup(fmt, q[i], table, n, lws[i], idx[i], stream=st)
            dn.ac_mx_fetch(fmt, table, n, idx[i], out[i], stream=st)
        torch.cuda.synchronize()
        values = dn.mx_dequantize(fmt, table, n, dim)
        for i in range(2):
            assert idx[i].tolist() == list(range(i, i + 80, 2)) and torch.equal(out[i], values[idx[i]]), rep


def test_the_longest_row():
    """2^31 - 32 values in a row are the blocks of as many rows of 32 values: the same bytes, and the same values."""
    cols, rows = 2 ** 31 - 32, 2 ** 26 - 1
    announce(f"mx row of {cols} values")
    x = torch.empty(cols, device=DEV, dtype=torch.bfloat16).normal_(generator=torch.Generator(device=DEV).manual_seed(3))
    for fmt in (dn.DN_MXFP4, dn.DN_MXFP8):
        a, b = dn.mx_quantize(fmt, x.view(1, cols)), dn.mx_quantize(fmt, x.view(rows, 32))
        used = rows * (17 if fmt == dn.DN_MXFP4 else 33)
        assert torch.equal(a[:used], b[:used])
        del b
        y = dn.mx_dequantize(fmt, a, 1, cols)
        for at in (0, 2 ** 30, cols - 2 ** 20):
            part = dn.mx_dequantize(fmt, dn.mx_quantize(fmt, x[at:at + 2 ** 20].view(-1, 32)), 2 ** 15, 32)
            assert torch.equal(y[0, at:at + 2 ** 20], part.view(-1)), at
        del a, y
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,N,K", [(33, 2 ** 22, 128), (3, 32, 2 ** 22)])
def test_the_widest_and_the_deepest_product(M, N, K):
    """Values of -1, 0 and 1, which the format holds: the sums are whole numbers below 2^24, exact in any order."""
    announce(f"mx4 linear {M}x{N}x{K}")
    g = torch.Generator(device=DEV).manual_seed(5)
    x, w = (torch.randint(-1, 2, (r, K), device=DEV, generator=g).float() for r in (M, N))
    y = torch.empty(M, N, device=DEV)
    dn.op_linear(F4, dn.mx_quantize(F4, x), dn.pack_weight(F4, w, N, K), None, y, M, N, K, y_f32=True)
    step = min(N, 2 ** 18)
    for at in range(0, N, step):
        assert torch.equal(y[:, at:at + step].double(), x.double() @ w[at:at + step].double().t().contiguous()), at
    del x, w, y
    torch.cuda.empty_cache()
