"""Microscaled 4-bit floating point from its definition, in numpy and fp64: the format's values, the quantiser's rule, the
product, and the packed byte order.  Nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TABLE = np.concatenate([MAGNITUDES, -MAGNITUDES])


def quantize(x: np.ndarray) -> tuple:
    """x [M, K], values of any type that are exact in fp64 -> (codes 0..15 [M, K] uint8, exponent bytes [M, K / 32] uint8)."""
    x = np.asarray(x, dtype=np.float64)
    M, K = x.shape
    b = x.reshape(M, K // 32, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    floor_log2 = np.frexp(top)[1] - 1                       # (frexp: top = f * 2^n with 1/2 <= f < 1)
    e = np.where(top == 0.0, 0, np.maximum(0, 125 + floor_log2))
    u = np.abs(b) * np.exp2(127.0 - e)[..., None]           # exact: fp64 holds every product of an input and this power of two
    d = np.abs(u[..., None] - MAGNITUDES)
    near = d == d.min(-1, keepdims=True)
    # of two magnitudes as near, the one with the even code
    code = np.where(near.sum(-1) == 1, near.argmax(-1), 0)
    for c in range(0, 8, 2):
        code = np.where((near.sum(-1) == 2) & near[..., c], c, code)
    code = code + 8 * np.signbit(b)
    e = np.where(bad, 255, e)
    return np.where(bad[..., None], 0, code).astype(np.uint8).reshape(M, K), e.astype(np.uint8)


def values(codes: np.ndarray, exponents: np.ndarray) -> np.ndarray:
    """fp64 values of codes [M, K] and exponent bytes [M, K / 32]; 255 is not a number."""
    M, K = codes.shape
    p = np.where(exponents == 255, np.nan, np.exp2(exponents.astype(np.float64) - 127.0))
    return (TABLE[codes].reshape(M, K // 32, 32) * p[..., None]).reshape(M, K)


def row_bytes(codes: np.ndarray) -> np.ndarray:
    """Codes [M, K] as the row form holds them: [M, K / 2] bytes, even columns in the low four bits."""
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def from_row_bytes(b: np.ndarray) -> np.ndarray:
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[0], -1)


def pack(codes: np.ndarray, exponents: np.ndarray) -> np.ndarray:
    """The packed form, byte by byte as it is specified."""
    N, K = codes.shape
    KT, KQ = K // 128, -(-K // 512)
    rec = KT * 1024 + KQ * 256
    out = np.zeros(N // 16 * rec, dtype=np.uint8)
    rows = row_bytes(codes)
    for n in range(N):
        rb, i = divmod(n, 16)
        for blk in range(K // 32):
            kt, o = divmod(blk, 4)
            lane = 16 * o + i
            at = rb * rec + kt * 1024 + 16 * lane
            out[at:at + 16] = rows[n, 16 * blk:16 * blk + 16]
            out[rb * rec + KT * 1024 + (kt // 4) * 256 + 4 * lane + kt % 4] = exponents[n, blk]
    return out


def product(x: np.ndarray, w: np.ndarray) -> tuple:
    """(X W^T, |X| |W|^T) in fp64 of dense fp64 values."""
    return x @ w.T, np.abs(x) @ np.abs(w).T
