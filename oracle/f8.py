"""Definition of the 8-bit floating-point layer in 64 bits (numpy): E4M3 elements, E8M0 scales per group of 128.

Elements are found by search in the table of the format's values, not by bit arithmetic; sums are numpy's in fp64.  Written
from the OCP format definitions and the operators' formulas; shares no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np

GROUP = 128
E4M3_MAX = 448.0


def e4m3_values() -> np.ndarray:
    """Values of the 256 bytes: sign, four exponent bits (bias 7), three mantissa bits; 0x7F and 0xFF are NaN, no infinities."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))
    v = np.where(b & 128, -v, v)
    v[[0x7F, 0xFF]] = np.nan
    return v


_POS = e4m3_values()[:127]  # ascending: 0 .. 448
_MID = (_POS[1:] + _POS[:-1]) / 2


def encode(v: np.ndarray) -> np.ndarray:
    """Nearest E4M3 byte, ties to the even one, saturating at 448; NaN -> 0x7F."""
    v = np.asarray(v, dtype=np.float64)
    a = np.minimum(np.abs(np.nan_to_num(v, nan=0.0, posinf=E4M3_MAX, neginf=E4M3_MAX)), E4M3_MAX)
    lo = np.searchsorted(_MID, a, side="left")  # a <= midpoint: the lower neighbour
    tie = (lo < _MID.size) & (a == _MID[np.minimum(lo, _MID.size - 1)])
    code = np.where(tie & (lo % 2 == 1), lo + 1, lo)
    code = np.where(np.signbit(v), code | 128, code)
    return np.where(np.isnan(v), 0x7F, code).astype(np.uint8)


def scale_byte(amax: np.ndarray) -> np.ndarray:
    """127 + the smallest e >= -127 with amax <= 448 * 2^e; 127 for zero."""
    amax = np.asarray(amax, dtype=np.float64)
    m, k = np.frexp(amax)  # amax = m * 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
    e = np.maximum(k - 9 + (m > 0.875), -127)
    return np.where(amax == 0, 127, e + 127).astype(np.int64)


def pow2(byte) -> np.ndarray:
    return np.ldexp(1.0, np.asarray(byte, dtype=np.int64) - 127)


def padded(K: int) -> int:
    return -(-K // GROUP) * GROUP


def pitch(K: int) -> int:
    return -(-K // (4 * GROUP)) * 4


def group_amax(v: np.ndarray) -> np.ndarray:
    """[M, K] -> [M, ceil(K / 128)], NaN left out."""
    M, K = v.shape
    p = np.zeros((M, padded(K)))
    p[:, :K] = np.nan_to_num(np.abs(v), nan=0.0, posinf=np.inf)
    return p.reshape(M, -1, GROUP).max(axis=2)


def quantize_rows(v: np.ndarray):
    """fp64 rows [M, K] -> codes uint8 [M, Kq], scale bytes uint8 [M, P]."""
    M, K = v.shape
    b = scale_byte(group_amax(v))
    p = np.zeros((M, padded(K)))
    p[:, :K] = v
    codes = encode(p / np.repeat(pow2(b), GROUP, axis=1))
    codes[:, K:] = 0
    scales = np.full((M, pitch(K)), 127, dtype=np.uint8)
    scales[:, : b.shape[1]] = b
    return codes, scales


def dequantize_rows(codes: np.ndarray, scales: np.ndarray, K: int) -> np.ndarray:
    s = np.repeat(pow2(scales[:, : codes.shape[1] // GROUP]), GROUP, axis=1)
    return (e4m3_values()[codes] * s)[:, :K]


def quantize_blocks(W: np.ndarray):
    """fp64 weights [N, K] -> codes uint8 [N, K], scale bytes uint8 [ceil(N / 128), ceil(K / 128)]."""
    N, K = W.shape
    g = np.zeros((padded(N), -(-K // GROUP)))
    g[:N] = group_amax(W)
    b = scale_byte(g.reshape(-1, GROUP, g.shape[1]).max(axis=1))
    s = np.repeat(np.repeat(pow2(b), GROUP, axis=0)[:N], GROUP, axis=1)[:, :K]
    return encode(W / s), b.astype(np.uint8)


def dequantize_blocks(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    N, K = codes.shape
    return e4m3_values()[codes] * np.repeat(np.repeat(pow2(scales), GROUP, axis=0)[:N], GROUP, axis=1)[:, :K]


def norm(x: np.ndarray, residual, gamma: np.ndarray, eps: float):
    """t = x + residual, y = t / sqrt(mean(t^2) + eps) * gamma."""
    t = x if residual is None else x + residual
    return t, t / np.sqrt((t * t).mean(axis=1, keepdims=True) + eps) * gamma


def silu(g: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g))
