"""Float64 oracle of the microscaled operands (TEST INFRASTRUCTURE ONLY, see the
package docstring): codes and scales of rows, the values that they stand for,
and the bytes of an operand in memory."""
from __future__ import annotations

import numpy as np

BLOCK = 32
TOP = {"e2m1": 6.0, "e4m3": 448.0}


def grid(fmt: str) -> np.ndarray:
    """The value of every code.  e2m1: sign, 2 exponent bits (bias 1), 1 mantissa
    bit; e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits, 0x7f and 0xff NaN."""
    ebits, mbits, bias = (2, 1, 1) if fmt == "e2m1" else (4, 3, 7)
    out = []
    for code in range(1 << (1 + ebits + mbits)):
        m, e, s = code & ((1 << mbits) - 1), (code >> mbits) & ((1 << ebits) - 1), code >> (ebits + mbits)
        v = m / (1 << mbits) * 2.0 ** (1 - bias) if e == 0 else (1 + m / (1 << mbits)) * 2.0 ** (e - bias)
        if fmt == "e4m3" and e == 15 and m == 7:
            v = np.nan
        out.append(-v if s else v)
    return np.array(out)


def nearest_codes(y: np.ndarray, fmt: str) -> np.ndarray:
    """Code bytes of code-unit values |y| <= top: nearest, ties to the even code, the sign of y."""
    half = grid(fmt)[:1 << (3 if fmt == "e2m1" else 7)]
    half = half[~np.isnan(half)]
    a = np.abs(y)
    up = np.clip(np.searchsorted(half, a), 1, len(half) - 1)
    lo, hi = a - half[up - 1], half[up] - a
    code = np.where((lo < hi) | ((lo == hi) & (up % 2 == 1)), up - 1, up)
    code = np.where(a == 0, 0, code)
    return (code + np.where(np.signbit(y), 8 if fmt == "e2m1" else 128, 0)).astype(np.uint8)


def quantize(x: np.ndarray, fmt: str):
    """Rows x (float64) -> code bytes [rows, blocks, 32] and scale bytes [rows, blocks]."""
    r, c = x.shape
    nb = -(-c // BLOCK)
    p = np.zeros((r, nb * BLOCK))
    p[:, :c] = x
    p = p.reshape(r, nb, BLOCK)
    bad = ~np.isfinite(p).all(-1)
    p = np.where(bad[..., None], 0.0, p)
    top = np.abs(p).max(-1)
    byte = np.zeros((r, nb), np.int64)                      # the smallest one whose top reaches the block's
    e = np.floor(np.log2(np.where(top > 0, top / TOP[fmt], 1.0))).astype(np.int64)
    for step in (-1, 0, 1, 2):                              # floor of a rounded logarithm, made sure of
        cand = e + step
        fits = (np.ldexp(TOP[fmt], cand) >= top) & (np.ldexp(TOP[fmt], cand - 1) < top)
        byte = np.where(fits, cand + 127, byte)
    byte = np.where(top > 0, np.maximum(byte, 0), 0)
    codes = nearest_codes(np.ldexp(p, (127 - byte)[..., None]), fmt)
    codes = np.where(bad[..., None], 0, codes).astype(np.uint8)
    return codes, np.where(bad, 255, byte).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray, fmt: str, cols: int) -> np.ndarray:
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (grid(fmt)[codes] * s[..., None]).reshape(codes.shape[0], -1)[:, :cols]


def unpack(buf: np.ndarray, fmt: str, rows: int, cols: int):
    """An operand's bytes -> (code bytes [rows, padded blocks, 32], scale bytes [rows, padded blocks])."""
    tiles, quads = -(-rows // 32), -(-cols // 256)
    per = 128 if fmt == "e2m1" else 256                     # bytes of 256 columns
    n = tiles * quads * 32 * per
    units = buf[:n].reshape(tiles, quads * per // 16, 32, 16).transpose(0, 2, 1, 3).reshape(tiles * 32, -1)
    codes = np.stack([units & 15, units >> 4], -1).reshape(tiles * 32, -1) if fmt == "e2m1" else units
    s = buf[n:n + tiles * quads * 256].reshape(tiles, quads, 2, 32, 4).transpose(0, 3, 1, 4, 2).reshape(tiles * 32, -1)
    return codes.reshape(tiles * 32, -1, BLOCK)[:rows], s[:rows]


def pack(codes: np.ndarray, scales: np.ndarray, fmt: str, fill: int = 0) -> np.ndarray:
    """The inverse of unpack for codes [rows, blocks, 32], scales [rows, blocks]; padding rows get ``fill``."""
    rows, nb = scales.shape
    tiles, quads = -(-rows // 32), -(-nb // 8)
    c = np.zeros((tiles * 32, quads * 8, BLOCK), np.uint8)
    s = np.zeros((tiles * 32, quads * 8), np.uint8)
    c[:rows, :nb], s[:rows, :nb] = codes, scales
    c[rows:], s[rows:] = fill & (15 if fmt == "e2m1" else 255), fill
    c = c.reshape(tiles * 32, -1)
    u = (c[:, 0::2] | (c[:, 1::2] << 4)) if fmt == "e2m1" else c
    u = u.reshape(tiles, 32, -1, 16).transpose(0, 2, 1, 3).reshape(-1)
    s = s.reshape(tiles, 32, quads, 4, 2).transpose(0, 2, 4, 1, 3).reshape(-1)
    return np.concatenate([u, s])
