"""Float64 oracle of the 8-bit KV cache's operators (TEST INFRASTRUCTURE ONLY,
see the package docstring): head norms, rotary positions, what a block's scale
and codes stand for, and attention over given keys and values."""
from __future__ import annotations

import math

import numpy as np

QMAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100


def code_values(fmt: str) -> np.ndarray:
    """The value of every code byte.  e4m3: sign, 4 exponent bits (bias 7), 3
    mantissa bits, no infinities, 0x7f and 0xff NaN."""
    b = np.arange(256)
    if fmt == "int8":
        return np.where(b < 128, b, b - 256).astype(np.float64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b < 128, v, -v)


def half_step(x: np.ndarray, fmt: str) -> np.ndarray:
    """Half the distance between neighbouring codes around the code-unit value x."""
    if fmt == "int8":
        return np.full_like(x, 0.5)
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def scale_needed(top: np.ndarray, fmt: str) -> np.ndarray:
    """The scale of a block whose largest magnitude is ``top``."""
    top = np.asarray(top, np.float64)
    s = top / QMAX[fmt]
    if fmt == "e4m3":
        s = np.where(top > 0, 2.0 ** np.ceil(np.log2(np.maximum(s, 1e-300))), 0.0)
    return np.where(top / QMAX[fmt] < TINY, 0.0, s)


def thetas(dim: int, base: float, scaling: str = "plain", factor: float = 1.0, low: float = 0.0, high: float = 0.0,
           orig_len: int = 0) -> np.ndarray:
    """Angle per position of each of the dim / 2 pairs."""
    out = []
    for i in range(dim // 2):
        b = base * factor ** (dim / (dim - 2)) if scaling == "ntk" else base
        t = math.exp(-2.0 * i / dim * math.log(b))
        if scaling == "linear":
            t /= factor
        if scaling == "bands":
            turns = orig_len * t / (2 * math.pi)
            w = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
            t = w * t + (1 - w) * t / factor
        out.append(t)
    return np.array(out)


def head_norm(x: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    return x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * gain


def rotate(x: np.ndarray, pos: np.ndarray, theta: np.ndarray, layout: str, mscale: float = 1.0) -> np.ndarray:
    """x [T, heads, dim]: its leading 2 len(theta) dims rotated by the rows' positions."""
    x = np.array(x, np.float64)
    n = len(theta)
    for t in range(x.shape[0]):
        for i in range(n):
            a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = mscale * math.cos(pos[t] * theta[i]), mscale * math.sin(pos[t] * theta[i])
            xa, xb = x[t, :, a].copy(), x[t, :, b].copy()
            x[t, :, a], x[t, :, b] = xa * c - xb * s, xa * s + xb * c
    return x


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One row: q [hd] over k, v [keys, hd]; the output, sum_j w_j |v_j| and
    the largest sum |q k| * scale of a key (for error bounds)."""
    s = k @ q * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ v, w @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * scale)
