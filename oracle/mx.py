"""Microscaled (MX) rows: the OCP Microscaling formats with 32-element blocks, E2M1 or E4M3
codes and one E8M0 scale per block (OCP Microscaling Formats (MX) Specification v1.0).

Test infrastructure only (see the package docstring).

Block scale byte s (2^(s - 127); 255 is NaN): max(floor(log2 max|x|) - e + 127, 0) with e the
exponent of the format's largest code (E2M1 6 = 1.5 * 2^2, E4M3 448 = 1.75 * 2^8), 0 for a block
of zeros, 255 for one that holds an infinity or a NaN. Code = x / 2^(s - 127) rounded to nearest,
ties to the even code, saturating.
"""

import numpy as np

BLOCK = 32
MXFP4, MXFP8 = 3, 4                 # the library's format numbers
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
                np.float64)
MAGNITUDES = {MXFP4: E2M1, MXFP8: E4M3}
EMAX = {MXFP4: 2, MXFP8: 8}
BLOCK_BYTES = {MXFP4: 16, MXFP8: 32}


def nearest(a, fmt):
    """Index of the magnitude nearest to a >= 0 (fp64), ties to the even index, saturating."""
    g = MAGNITUDES[fmt]
    hi = np.clip(np.searchsorted(g, a, side="left"), 1, len(g) - 1)
    lo = hi - 1
    dl, dh = a - g[lo], g[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(a >= g[-1], len(g) - 1, np.where(up, hi, lo))


def scales(x, fmt):
    """Scale bytes [rows, blocks] of rows x [rows, blocks * 32] (fp64 values)."""
    a = np.abs(x).reshape(x.shape[0], -1, BLOCK).max(2)
    with np.errstate(invalid="ignore"):
        e = np.frexp(np.where(np.isfinite(a), a, 1.0))[1] - 1
    s = np.where(a > 0, np.maximum(e - EMAX[fmt] + 127, 0), 0)
    return np.where(np.isfinite(np.abs(x).reshape(x.shape[0], -1, BLOCK)).all(2), s, 255).astype(np.uint8)


def quantize(x, fmt):
    """Rows x [rows, cols] -> (codes [rows, B * 32] one per byte, scales [rows, B])."""
    x = np.asarray(x, np.float64)
    pad = -x.shape[1] % BLOCK
    x = np.concatenate([x, np.zeros((x.shape[0], pad))], 1)
    s = scales(x, fmt)
    v = x * np.repeat(2.0 ** (127.0 - s), BLOCK, axis=1)
    bad = np.repeat(s == 255, BLOCK, axis=1)
    idx = nearest(np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0))), fmt)
    sign = np.where(np.signbit(v) & ~bad, len(MAGNITUDES[MXFP4]) if fmt == MXFP4 else 128, 0)
    return (idx + sign).astype(np.uint8), s


def values(codes, s, fmt, cols):
    """The values [rows, cols] (fp64) that codes and scales stand for."""
    half = 8 if fmt == MXFP4 else 128
    g = np.concatenate([MAGNITUDES[fmt], np.full(half - len(MAGNITUDES[fmt]), np.nan)])
    v = np.where(codes >= half, -1.0, 1.0) * g[codes % half]
    k = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return (v * np.repeat(k, BLOCK, axis=1))[:, :cols]


def rounded(x, fmt):
    """The values rows x become in the format."""
    x = np.asarray(x, np.float64)
    return values(*quantize(x, fmt), fmt, x.shape[1])


def n_bytes(fmt, rows, cols):
    b = -(-cols // BLOCK)
    return rows * b * BLOCK_BYTES[fmt] + -(-rows * b // 16) * 16 + 16


def to_buffer(codes, s, fmt):
    """Codes and scales as the bytes of an MX buffer (without its padding)."""
    if fmt == MXFP4:
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return np.concatenate([codes.reshape(-1), s.reshape(-1)]).astype(np.uint8)


def from_buffer(buf, fmt, rows, cols):
    """(codes, scales) of an MX buffer."""
    b = -(-cols // BLOCK)
    n = rows * b * BLOCK_BYTES[fmt]
    c = buf[:n].reshape(rows, -1)
    if fmt == MXFP4:
        c = np.stack([c & 15, c >> 4], 2).reshape(rows, -1)
    return c, buf[n:n + rows * b].reshape(rows, b)


def mx4_model_weights(W):
    """The 4-bit variant's parameters: the bf16 model's except the feed-forward matrices, which
    are quantised along their input dimension from the fp32 draws (the values they become)."""
    from .unet import bf16_model_weights
    out = bf16_model_weights(W)
    for k, v in W.items():
        if k.endswith(".ff1.w") or k.endswith(".ff2.w"):
            out[k] = rounded(v, MXFP4).astype(np.float32)
    return out


def mx4_act(x):
    """A feed-forward input [..., C] in 4-bit rows, as fp32."""
    x = np.asarray(x)
    return rounded(x.reshape(-1, x.shape[-1]), MXFP4).reshape(x.shape).astype(np.float32)
