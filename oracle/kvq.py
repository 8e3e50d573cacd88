"""Oracle of the 8-bit KV cache and of attention with error bounds: plain numpy in fp64, from the definitions.

A block is 16 positions of one head with one scale s.  e4m3: s is the smallest power of two with max|x| <= 448 s and a value
is s times the nearest e4m3 number to x / s (ties to even; s is at most 2^119, beyond 448 * 2^119 the largest number is taken); int8: s = max|x| / 127 rounded to fp32, value s * round(x / s).
Scales are at least 2^-100; a block of zeros is zeros under any s (here 1; a cache holds it with the smallest); NaN and infinities count as 0.  Positions of the incomplete last
block keep their values.  The paper (Sec. 3.3) keeps bf16 caches; the arithmetic here is this library's definition.
"""
from __future__ import annotations

import numpy as np

BLOCK = 16
MIN_SCALE = 2.0 ** -100


def scale(amax: float, fmt: str) -> float:
    if amax == 0.0:
        return 1.0
    if fmt == "int8":
        return max(float(np.float32(amax / 127.0)), MIN_SCALE)
    e = -100
    while amax > 448.0 * 2.0 ** e and e < 119:
        e += 1
    return 2.0 ** e


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """Nearest e4m3 number (ties to even) of |y| <= 448: three fraction bits, smallest normal exponent -6, subnormals below."""
    _, e = np.frexp(np.maximum(np.abs(y), 2.0 ** -6))     # |y| = m 2^e, m in [0.5, 1)
    step = np.ldexp(1.0, e - 1 - 3)
    return np.rint(y / step) * step


def block_values(x: np.ndarray, fmt: str) -> np.ndarray:
    """Values the codes of one block x [16][D] (one head) stand for."""
    s = scale(float(np.abs(x).max()), fmt)
    return round_e4m3(np.clip(x / s, -448, 448)) * s if fmt == "e4m3" else np.clip(np.rint(x / s), -127, 127) * s


def cache_values(x: np.ndarray, fmt: str) -> np.ndarray:
    """What a cache filled with the rows x [n][H][D] holds."""
    y = np.where(np.isfinite(x), x, 0.0).astype(np.float64)
    for j in range(len(y) // BLOCK):
        for h in range(y.shape[1]):
            y[j * BLOCK:(j + 1) * BLOCK, h] = block_values(y[j * BLOCK:(j + 1) * BLOCK, h], fmt)
    return y


def key_scales(x: np.ndarray, fmt: str) -> np.ndarray:
    """Scale that the block of each position of x [n][H][D] is held with, [n][H] (a block of zeros, whose codes are zeros under any
    scale: the smallest); 0 in the incomplete last block."""
    y = np.where(np.isfinite(x), x, 0.0)
    out = np.zeros(x.shape[:2])
    for j in range(len(y) // BLOCK):
        for h in range(y.shape[1]):
            amax = float(np.abs(y[j * BLOCK:(j + 1) * BLOCK, h]).max())
            out[j * BLOCK:(j + 1) * BLOCK, h] = scale(amax, fmt) if amax > 0 else MIN_SCALE
    return out


def kept(n: int, fa: bool, S: int, W: int) -> np.ndarray:
    """Positions a decode step at length n attends to (Eq. 1, or Eq. 2 with sink and window)."""
    j = np.arange(n)
    return j if fa else j[(j < S) | (j >= n - W)]


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale_: float):
    """softmax(scale q k^T) v for q [Hq][D] over k, v [m][Hkv][D] -> (out [Hq][D], sum_j p_j |v_j| [Hq][D],
    max_j scale * sum_d |q_d k_jd| [Hq], p [Hq][m])."""
    G = q.shape[0] // k.shape[1]
    kk, vv = np.repeat(k, G, axis=1), np.repeat(v, G, axis=1)
    s = np.einsum("hd,mhd->hm", q, kk) * scale_
    p = np.exp(s - s.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    mag = (np.einsum("hd,mhd->hm", np.abs(q), np.abs(kk)) * scale_).max(axis=1)
    return np.einsum("hm,mhd->hd", p, vv), np.einsum("hm,mhd->hd", p, np.abs(vv)), mag, p
