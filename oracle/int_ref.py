"""Reference of the linear layers in 8-bit integers -- TEST INFRASTRUCTURE ONLY.

Rows y become codes q and a scale: with m = max|y|, scale = fl32(m / 127) and q the
whole number nearest to 127 y / m, ties to even; m = 0 gives zeros and scale 0; a row
with an infinity or a NaN gives zero codes and a NaN scale.  A product of codes is
z = (sum_k qx qw) sx sw + bias, exact up to fp64.

Pins (tests/test_int.py): rows decided in rational arithmetic, worked ties, quantising
values that codes stand for gives the codes back, products by scalar loops.
"""
from __future__ import annotations

import numpy as np

from .ardit_ref import gelu_tanh, rms_norm  # noqa: F401


def quantize(y):
    """(codes int8, scales fp32, margin) of rows y; margin is how far 127 |y| / m lies from the
    nearest half (borders that fp64 arithmetic before this cannot decide have margins near 0)."""
    y = np.asarray(y, np.float64)
    a = np.abs(y)
    m = a.max(-1)
    bad = ~np.isfinite(y).all(-1)
    live = (m > 0) & ~bad
    unit = np.where(live, m, 1.0)[..., None]
    a = np.where(live[..., None], a, 0.0)
    k = np.floor(127.0 * (a / unit))
    side = 254.0 * a - (2.0 * k + 1.0) * unit
    up = (side > 0) | ((side == 0) & (k % 2 == 1))
    codes = np.where(np.signbit(y), -(k + up), k + up).astype(np.int8)
    with np.errstate(invalid="ignore"):
        scales = np.where(bad, np.nan, m / 127.0).astype(np.float32)
    return codes, scales, np.abs(side) / (2.0 * unit)


def dequantize(codes, scales):
    """Values of codes in fp64."""
    return np.asarray(codes, np.float64) * np.asarray(scales, np.float64)[..., None]


def norm(h, eps, gain=None, scale=None, shift=None):
    """y of rows h (fp64): rms(h) * gain, or * (1 + scale) + shift (per row or shared)."""
    h = np.asarray(h, np.float64)
    u = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    if gain is not None:
        return u * np.asarray(gain, np.float64)
    if scale is not None:
        u = u * (1.0 + np.asarray(scale, np.float64))
    return u if shift is None else u + np.asarray(shift, np.float64)


def product(qx, sx, qw, sw):
    """(sum_k qx qw) sx sw in fp64 (sums exact)."""
    s = np.asarray(qx, np.float64) @ np.asarray(qw, np.float64).T
    return s * np.asarray(sx, np.float64)[:, None] * np.asarray(sw, np.float64)[None, :]


def linear(qx, sx, qw, sw, bias=None, gelu=False, res=None, gate=None):
    """(result, product part) in fp64; gate per row and column."""
    p = product(qx, sx, qw, sw)
    z = p if bias is None else p + np.asarray(bias, np.float64)
    if gelu:
        return gelu_tanh(z), p
    if res is not None:
        z = np.asarray(res, np.float64) + (z if gate is None else np.asarray(gate, np.float64) * z)
    return z, p


def quantized_linear(x, qw, sw, bias):
    """x (rows, fp64) quantised per row, then through codes qw with scales sw."""
    qx, sx, _ = quantize(x)
    return linear(qx, sx, qw, sw, bias)[0]
