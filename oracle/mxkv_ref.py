"""Reference of the microscaled key/value cache -- TEST INFRASTRUCTURE ONLY.

Keys and values held in E4M3 (8 bits) or E2M1 (4 bits) in blocks of 32 along
each attention product's summed axis, with a power of two 2^e per block:
  - keys: 32 consecutive dims of a token's head;
  - values: 32 consecutive keys of one page, per dim (a page's last block may
    hold fewer);
  - e is the smallest exponent, at least -117, with max|x| / 2^e below 256
    (E4M3) or at most 6 (E2M1), there at most 125 (6 2^126 is past bf16); an
    all-zero block takes -117; a block with an infinity or NaN reads back as NaN;
  - codes are the nearest values of the format, ties to the even code.

A page of T tokens lies in tiles of 64 keys (T64 = T rounded up): k_codes
[H][T64][d], k_scales [H][T64][d / 32], v_codes [H][T64 / 64][d][64], v_scales
[H][T64 / 64][2][d]; scale bytes are e + 127 (255: NaN).

Pins (tests/test_kvmx.py): the formats' values from their definitions, worked
ties, the exponent's definition by search, exactly representable blocks pass
unchanged, errors within half a step, pack and unpack are inverse.
"""
from __future__ import annotations

import numpy as np

from .ardit_ref import rms_norm, rope3d  # noqa: F401  (the append's arithmetic)
from .fp8_ref import e4m3_values

BLOCK = 32
MIN_EXP = -117


def grid(bits: int) -> np.ndarray:
    """The format's non-negative finite values in code order."""
    if bits == 8:
        return e4m3_values()[:127]
    vals = []
    for code in range(8):
        ex, m = code >> 1, code & 1
        vals.append(m * 0.5 if ex == 0 else (1 + m / 2.0) * 2.0 ** (ex - 1))
    return np.array(vals)


def exponent(amax, bits: int):
    """Smallest e >= -117 with amax / 2^e < 256 (8 bits) or <= 6 (4 bits, e <= 125)."""
    amax = np.asarray(amax, np.float64)
    m, ex = np.frexp(np.where(amax > 0, amax, 1.0))       # amax = m 2^ex, m in [0.5, 1)
    e = ex - 8 if bits == 8 else np.minimum(np.where(m <= 0.75, ex - 3, ex - 2), 125)
    return np.where(amax > 0, np.maximum(e, MIN_EXP), MIN_EXP).astype(np.int64)


def encode(x, e, bits: int):
    """Codes (sign in the top bit) of x / 2^e, nearest, ties to the even code."""
    g = grid(bits)
    a = np.abs(np.asarray(x, np.float64)) / np.ldexp(1.0, e)
    hi = np.clip(np.searchsorted(g, a), 1, len(g) - 1)
    lo = hi - 1
    below, above = a - g[lo], g[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    return np.where(np.signbit(x), code + (1 << (bits - 1)), code).astype(np.uint8)


def decode(codes, e, bits: int):
    g = grid(bits)
    sign = 1 << (bits - 1)
    c = np.asarray(codes).astype(np.int64)
    v = np.where(c & sign, -1.0, 1.0) * g[np.minimum(c & (sign - 1), len(g) - 1)]
    return v * np.ldexp(1.0, e)


def quantize(x, bits: int, axis: int = -1):
    """(codes, e per element) in blocks of 32 along axis, the last maybe short."""
    x = np.moveaxis(np.asarray(x, np.float64), axis, -1)
    n = x.shape[-1]
    pad = -n % BLOCK
    xp = np.concatenate([x, np.zeros(x.shape[:-1] + (pad,))], -1)
    xb = xp.reshape(x.shape[:-1] + (-1, BLOCK))
    bad = ~np.isfinite(xb).all(-1)
    e = exponent(np.where(bad, 0.0, np.abs(np.where(np.isfinite(xb), xb, 0.0)).max(-1)), bits)
    codes = encode(np.where(np.isfinite(xb), xb, 0.0), e[..., None], bits)
    e = np.where(bad, 128, e)
    e = np.broadcast_to(e[..., None], xb.shape).reshape(xp.shape)[..., :n]
    codes = codes.reshape(xp.shape)[..., :n]
    return np.moveaxis(codes, -1, axis), np.moveaxis(e, -1, axis)


def rounded(x, bits: int, axis: int = -1):
    """The values that x's codes stand for."""
    codes, e = quantize(x, bits, axis)
    return np.where(e == 128, np.nan, decode(codes, np.where(e == 128, 0, e), bits))


class Pages:
    """Host image of a pool, bytes filled with `fill` where nothing was packed."""

    def __init__(self, n_pages, H, d, T, bits, fill=0xFF):
        self.H, self.d, self.T, self.bits = H, d, T, bits
        self.nt = (T + 63) // 64
        per = 8 // bits
        self.k_codes = np.full((n_pages, H, 64 * self.nt, d // per), fill, np.uint8)
        self.k_scales = np.full((n_pages, H, 64 * self.nt, d // 32), fill, np.uint8)
        self.v_codes = np.full((n_pages, H, self.nt, d, 64 // per), fill, np.uint8)
        self.v_scales = np.full((n_pages, H, self.nt, 2, d), fill, np.uint8)

    def _bytes(self, codes):
        return codes if self.bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)

    def _codes(self, b):
        if self.bits == 8:
            return b
        return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))

    def pack(self, page, k, v):
        """k, v [n, H, d], n <= T tokens of one page; returns the values they become."""
        n = k.shape[0]
        kc, ke = quantize(k, self.bits, -1)
        vc, ve = quantize(v, self.bits, 0)
        self.k_codes[page, :, :n] = self._bytes(kc.transpose(1, 0, 2))
        self.k_scales[page, :, :n] = (ke[:, :, ::BLOCK] + 127).transpose(1, 0, 2)
        tiles = (self.H, 64 * self.nt, self.d)
        flat = self._codes(self.v_codes[page]).transpose(0, 1, 3, 2).reshape(tiles).copy()
        flat[:, :n] = vc.transpose(1, 0, 2)
        self.v_codes[page] = self._bytes(flat.reshape(self.H, self.nt, 64, self.d).transpose(0, 1, 3, 2))
        blocks = self.v_scales[page].reshape(self.H, 2 * self.nt, self.d)
        blocks[:, :(n + BLOCK - 1) // BLOCK] = (ve[::BLOCK] + 127).transpose(1, 0, 2)
        return (decode_nan(kc, ke, self.bits), decode_nan(vc, ve, self.bits))

    def unpack(self, page, n=None):
        """Values (k, v) [n, H, d] of a page's first n tokens."""
        n = self.T if n is None else n
        ke = self.k_scales[page].astype(np.int64).repeat(BLOCK, -1) - 127      # [H, T64, d]
        k = decode_nan(self._codes(self.k_codes[page]), ke, self.bits).transpose(1, 0, 2)
        ve = self.v_scales[page].astype(np.int64).transpose(0, 1, 3, 2).repeat(BLOCK, -1) - 127
        v = decode_nan(self._codes(self.v_codes[page]), ve, self.bits)         # [H, nt, d, 64]
        v = v.transpose(1, 3, 0, 2).reshape(64 * self.nt, self.H, self.d)
        return k[:n], v[:n]


def decode_nan(codes, e, bits):
    """decode with the NaN scale, and E4M3's NaN codes."""
    bad = np.asarray(e) == 128
    if bits == 8:
        bad = bad | ((np.asarray(codes) & 0x7F) == 0x7F)
    return np.where(bad, np.nan, decode(codes, np.where(np.asarray(e) == 128, 0, e), bits))
