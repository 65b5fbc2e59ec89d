"""Pins of the oracle's microscaled rows (oracle.mx): code values written out by hand, every
midpoint, brute-force nearest values, torch's E4M3 conversion, block scales at powers of two,
zero, subnormal and non-finite blocks, and the buffer layout."""

import numpy as np
import pytest
import torch

from oracle import mx, topology as T, unet as U
from paper_2511_06724_amd import workloads as W


def test_magnitudes():
    assert list(mx.E2M1) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(mx.E4M3, t)


@pytest.mark.parametrize("fmt", [mx.MXFP4, mx.MXFP8])
def test_nearest_midpoints_and_neighbours(fmt):
    g = mx.MAGNITUDES[fmt]
    assert np.array_equal(mx.nearest(g, fmt), np.arange(len(g)))
    mid = (g[:-1] + g[1:]) / 2
    even = np.arange(len(g) - 1) + np.arange(len(g) - 1) % 2
    assert np.array_equal(mx.nearest(mid, fmt), even)
    assert np.array_equal(mx.nearest(np.nextafter(mid, 0), fmt), np.arange(len(g) - 1))
    assert np.array_equal(mx.nearest(np.nextafter(mid, 1e9), fmt), np.arange(1, len(g)))
    assert list(mx.nearest(np.array([g[-1] * 1.01, 1e30]), fmt)) == [len(g) - 1] * 2


def test_blocks_by_hand():
    x = np.zeros((1, 40))
    x[0, :5] = [4.0, -3.5, 0.25, 0.75, 7.99]      # largest 7.99: scale 2^0; ties to even, 7.99 saturates
    x[0, 32:35] = [2.0 ** -20, -(2.0 ** -21), 0.0]
    c, s = mx.quantize(x, mx.MXFP4)
    assert list(s[0]) == [127, 127 - 22]
    assert list(mx.values(c, s, mx.MXFP4, 40)[0, :5]) == [4.0, -4.0, 0.0, 1.0, 6.0]
    assert list(mx.values(c, s, mx.MXFP4, 40)[0, 32:35]) == [2.0 ** -20, -(2.0 ** -21), 0.0]
    assert c.shape == (1, 64) and not c[0, 40:].any()


@pytest.mark.parametrize("fmt", [mx.MXFP4, mx.MXFP8])
def test_special_blocks(fmt):
    x = np.zeros((6, 32))
    x[1, 3] = np.inf
    x[2, 31] = np.nan
    x[3, 0] = 1e-45                                # below every scale
    x[4, :] = np.finfo(np.float32).max
    x[5, 0] = -np.finfo(np.float32).max
    c, s = mx.quantize(x, fmt)
    v = mx.values(c, s, fmt, 32)
    assert list(s[:4, 0]) == [0, 255, 255, 0] and s[4, 0] == s[5, 0] == 254 - mx.EMAX[fmt]
    assert not v[0].any() and np.isnan(v[1]).all() and np.isnan(v[2]).all()
    assert (v[4] == mx.MAGNITUDES[fmt][-1] * 2.0 ** (127 - mx.EMAX[fmt])).all() and v[5, 0] == -v[4, 0]


def test_scale_at_powers_of_two():
    for e in (-126, -30, -1, 0, 1, 60, 127):
        for a, want in ((2.0 ** e, e), (np.nextafter(np.float32(2.0 ** e), np.float32(0)), e - 1)):
            x = np.zeros((1, 32))
            x[0, 7] = a
            assert mx.scales(x, mx.MXFP4)[0, 0] == max(want - 2 + 127, 0)
            assert mx.scales(x, mx.MXFP8)[0, 0] == max(want - 8 + 127, 0)


def test_rounded_against_brute_force_and_torch():
    r = np.random.default_rng(5)
    x = (r.standard_normal((20, 96)) * 2.0 ** r.integers(-20, 20, (20, 1))).astype(np.float32)
    for fmt in (mx.MXFP4, mx.MXFP8):
        _, s = mx.quantize(x, fmt)
        k = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=1)
        grid = np.concatenate([mx.MAGNITUDES[fmt], -mx.MAGNITUDES[fmt]])
        best = np.abs(x[:, :, None] / k[:, :, None] - grid).min(2)
        assert np.array_equal(np.abs(mx.rounded(x, fmt) - x) / k, best)
    t = torch.from_numpy((x / k).astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(mx.rounded(x, mx.MXFP8) / k, t)


@pytest.mark.parametrize("fmt", [mx.MXFP4, mx.MXFP8])
def test_buffer_layout(fmt):
    x = np.random.default_rng(1).standard_normal((3, 45))
    c, s = mx.quantize(x, fmt)
    b = mx.to_buffer(c, s, fmt)
    assert b.size <= mx.n_bytes(fmt, 3, 45) < b.size + 32
    c2, s2 = mx.from_buffer(b, fmt, 3, 45)
    assert np.array_equal(c, c2) and np.array_equal(s, s2)
    assert b[0] == (c[0, 0] | (c[0, 1] << 4) if fmt == mx.MXFP4 else c[0, 0])


def test_mx4_model_weights_touch_only_the_feed_forward():
    cfg = W.tiny(W.DN_MXFP4).with_(model_channels=128, levels=((128, 1, 4, 32),))
    table = [(int(np.prod(sh)), f, k) for _, sh, k, f in T.tensor_table(cfg)]
    Wt = U.unpack(cfg, W.weight_blob(table, 3))
    W4, W16 = mx.mx4_model_weights(Wt), U.bf16_model_weights(Wt)
    ff = [k for k in Wt if k.endswith(".ff1.w") or k.endswith(".ff2.w")]
    assert len(ff) == 2
    for k in Wt:
        assert np.array_equal(W4[k], mx.rounded(Wt[k], mx.MXFP4) if k in ff else W16[k])
