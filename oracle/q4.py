"""64-bit implementation of the 4-bit weights, in numpy, from their definition."""
import numpy as np


def bf16(x):
    """float64 values rounded to bf16 (half to even), as float64; finite values within the range of bf16."""
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0))), 0.0)
    e = np.where(a >= 2.0 ** (e + 1), e + 1, np.where(a < 2.0 ** e, e - 1, e))   # log2 may be off next to a power of two
    step = 2.0 ** (np.maximum(e, -126) - 7)
    return np.rint(x / step) * step


def quantize(W, G):
    """(q int [K][N], scales float64 [groups][N]); a group with an infinity or NaN has scale NaN and codes 0."""
    K, N = W.shape
    q, s = np.zeros((K, N), np.int64), np.zeros(((K + G - 1) // G, N))
    for g in range(s.shape[0]):
        w = W[g * G:(g + 1) * G]
        fine = np.isfinite(w).all(axis=0)
        s[g] = np.where(fine, bf16(np.where(fine, np.abs(w).max(axis=0), 0.0) / 7), np.nan)
        ok = fine & (s[g] > 0)
        q[g * G:(g + 1) * G][:, ok] = np.clip(np.rint(w[:, ok] / s[g, ok]), -7, 7).astype(np.int64)
    return q, s


def pack(q):
    """codes uint8 [K / 2][N]."""
    return ((q[0::2] & 15) | (q[1::2] & 15) << 4).astype(np.uint8)


def unpack(codes):
    q = np.empty((2 * codes.shape[0], codes.shape[1]), np.int64)
    q[0::2], q[1::2] = codes & 15, codes >> 4
    return np.where(q >= 8, q - 16, q)


def values(q, scales, G):
    return q * np.repeat(scales, G, axis=0)[: q.shape[0]]
