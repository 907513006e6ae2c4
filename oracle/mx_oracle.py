"""Microscaled (MX) blocks in plain fp64 NumPy: quantisation, its meaning, the operators on it.  Test infrastructure only; written from the
definition in include/dartqr.h and sharing no code with the library.

A row is cut into blocks of 32 values.  Of a block whose largest magnitude is a, E = max(floor(log2 a) - e, -127) with e the exponent of the
largest representable value; a value becomes 2^E times the representable value nearest to v / 2^E, ties to the even code, clamped.
"""

from __future__ import annotations

import numpy as np

MXFP4, MXFP8 = 0, 1


def grid(fmt: int) -> np.ndarray:
    """Representable magnitudes in the order of their codes (e4m3 without its NaN)."""
    mant, bias, count = (1, 1, 8) if fmt == MXFP4 else (3, 7, 127)
    code = np.arange(count)
    exp, frac = code >> mant, code & ((1 << mant) - 1)
    return np.where(exp == 0, frac * 2.0 ** (1 - bias - mant), ((1 << mant) + frac) * 2.0 ** (exp - bias - mant + 0.0))


def blocks(n: int) -> int:
    return -(-n // 32)


def quantize(X: np.ndarray, fmt: int):
    """(codes T x 32 blocks, unpacked, one an entry; scale bytes T x blocks) of the rows of X."""
    X = np.asarray(X, dtype=np.float64)
    T, n = X.shape
    nb = blocks(n)
    V = np.zeros((T, nb * 32))
    V[:, :n] = X
    V = V.reshape(T, nb, 32)
    levels = grid(fmt)
    bad = ~np.isfinite(V).all(-1)
    V = np.where(bad[..., None], 0.0, V)
    top = np.abs(V).max(-1)
    floor_log2 = np.frexp(top)[1] - 1.0                                  # top = m 2^k with 0.5 <= m < 1
    E = np.where(top > 0, np.maximum(floor_log2 - (2 if fmt == MXFP4 else 8), -127), -127)
    A = np.abs(V) / 2.0 ** E[..., None]
    mid = (levels[1:] + levels[:-1]) / 2
    code = np.searchsorted(mid, A, side="left")                          # a tie stays below
    tie = (code < mid.size) & (mid[np.minimum(code, mid.size - 1)] == A)
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    sign = np.signbit(V) * (8 if fmt == MXFP4 else 128)
    codes = np.where(bad[..., None], 0, code + sign).astype(np.uint8).reshape(T, nb * 32)
    return codes, np.where(bad, 255, E + 127).astype(np.uint8)


def pack(codes: np.ndarray, fmt: int) -> np.ndarray:
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8) if fmt == MXFP4 else codes


def unpack(data: np.ndarray, fmt: int) -> np.ndarray:
    if fmt == MXFP8:
        return data
    out = np.empty((data.shape[0], data.shape[1] * 2), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = data & 15, data >> 4
    return out


def values(codes: np.ndarray, scales: np.ndarray, n: int, fmt: int) -> np.ndarray:
    """What unpacked codes and their scale bytes stand for."""
    levels = grid(fmt)
    table = np.concatenate([levels, -levels]) if fmt == MXFP4 else np.concatenate([levels, [np.nan], -levels, [np.nan]])
    T, nb = scales.shape
    with np.errstate(invalid="ignore"):
        per = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return (table[codes].reshape(T, nb, 32) * per[..., None]).reshape(T, nb * 32)[:, :n]


def through(X: np.ndarray, fmt: int) -> np.ndarray:
    codes, scales = quantize(X, fmt)
    return values(codes, scales, X.shape[1], fmt)


def rms_norm(h: np.ndarray, gain, eps: float) -> np.ndarray:
    """h / sqrt(mean h^2 + eps) * gain row by row; a row whose root vanishes gives zeros."""
    h = np.asarray(h, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        root = np.sqrt((h * h).mean(-1, keepdims=True) + float(np.float32(eps)))
        y = np.where(root == 0, 0.0, h / np.where(root == 0, 1.0, root))
        return y if gain is None else y * np.asarray(gain, dtype=np.float64)


def objective(Y: np.ndarray, fmt: int, reduce: str = "mean"):
    """Loss (1/n) sum (y - yhat)^2, combined over the rows, and its derivative with yhat held fixed."""
    Y = np.asarray(Y, dtype=np.float64)
    T, n = Y.shape
    c = 1.0 / T if reduce == "mean" else 1.0
    e = Y - through(Y, fmt)
    return c * (e * e).sum() / n, c * 2.0 / n * e
