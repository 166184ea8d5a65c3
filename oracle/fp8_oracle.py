"""8-bit floating point with a scale for each block of 128, and the gated block on it, from their definitions, in numpy and fp64.
Nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

FLOOR = 2.0 ** -110


def _value(code: int) -> float:
    sign, e, m = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return float("nan")
    return sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))


TABLE = np.array([_value(c) for c in range(256)])
MAGNITUDES = TABLE[:127]                                 # ascending; code 126 is 448


def codes_of(u: np.ndarray) -> np.ndarray:
    """The nearest code to each finite value, ties to the even code, 448 beyond it."""
    a = np.abs(u)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 126)      # MAGNITUDES[hi - 1] <= a <= MAGNITUDES[hi], where 448 is not passed
    below, above = a - MAGNITUDES[hi - 1], MAGNITUDES[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return (np.where(up, hi, hi - 1) + 128 * np.signbit(u)).astype(np.uint8)


def _block(x: np.ndarray, axes, power: bool = False) -> tuple:
    """Codes of fp64 blocks that share a scale along `axes`, and the scales (fp32, those axes kept)."""
    bad = ~np.isfinite(x).all(axes, keepdims=True)
    x = np.where(bad, np.copysign(0.0, 1.0), x)
    a = np.maximum(np.abs(x).max(axes, keepdims=True), FLOOR)
    if power:
        f, e = np.frexp(a)                                    # a = f 2^e, 1/2 <= f < 1; 448 = 0.875 * 2^9
        s = np.exp2(np.where(f <= 0.875, e - 9, e - 8).astype(np.float64))
        u = x / s
    else:
        s, r = (a / 448.0).astype(np.float32), (448.0 / a).astype(np.float32)
        u = (x * r.astype(np.float64)).astype(np.float32).astype(np.float64)     # (24 bits by 24: exact in fp64)
    return np.where(bad, 0, codes_of(u)).astype(np.uint8), np.where(bad, np.nan, s).astype(np.float32)


def quantize_rows(x: np.ndarray) -> tuple:
    """x [M, K] -> codes [M, K], scales [K / 128, M]."""
    M, K = x.shape
    c, s = _block(np.asarray(x, np.float64).reshape(M, K // 128, 128), (2,))
    return c.reshape(M, K), s[..., 0].T.copy()


def quantize_weights(w: np.ndarray) -> tuple:
    """w [N, K] -> codes [N, K], scales [ceil(N / 128), K / 128]."""
    N, K = w.shape
    p = np.zeros((-(-N // 128) * 128, K))
    p[:N] = w
    c, s = _block(p.reshape(-1, 128, K // 128, 128), (1, 3))
    return c.reshape(-1, K)[:N].copy(), s[:, 0, :, 0].copy()


def quantize_columns(x: np.ndarray) -> tuple:
    """x [M, K] -> codes [K, M'], scales [M' / 128, K]."""
    M, K = x.shape
    p = np.zeros((-(-M // 128) * 128, K))
    p[:M] = x
    c, s = _block(p.reshape(-1, 128, K), (1,), power=True)
    return c.reshape(-1, K).T.copy(), s[:, 0, :].copy()


def row_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    M, K = codes.shape
    return (TABLE[codes].reshape(M, K // 128, 128) * scales.astype(np.float64).T[..., None]).reshape(M, K)


def weight_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    N, K = codes.shape
    return TABLE[codes] * np.repeat(np.repeat(scales.astype(np.float64), 128, 0)[:N], 128, 1)


def product(x: np.ndarray, w: np.ndarray) -> tuple:
    """(X W^T, |X| |W|^T) in fp64 of dense fp64 values."""
    return x @ w.T, np.abs(x) @ np.abs(w).T


def argument(g: np.ndarray, act: str) -> np.ndarray:
    return g if act == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)


def sigma(z: np.ndarray) -> np.ndarray:
    """1 / (1 + exp(-z)), which is (1 + tanh(z / 2)) / 2, without cancellation at either end."""
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def activation(g: np.ndarray, act: str) -> np.ndarray:
    return g * sigma(argument(g, act))


def slope(g: np.ndarray, act: str) -> np.ndarray:
    """Its derivative."""
    z = argument(g, act)
    dz = 1.0 if act == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (1.0 + 3 * 0.044715 * g * g)
    return sigma(z) * (1.0 + g * sigma(-z) * dz)


def gated_gradients(dh: np.ndarray, g: np.ndarray, u: np.ndarray, act: str) -> tuple:
    return dh * u * slope(g, act), dh * activation(g, act)
