"""Plain NumPy definitions of the microscaled 4-bit rows, in float64 (test
infrastructure; the definitions are those of ``include/gcn_rows4.h``)."""
from __future__ import annotations

import numpy as np

BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TABLE = np.concatenate([MAGNITUDES, -MAGNITUDES])


def exponent(a: float) -> int:
    """Scale exponent of a block whose largest magnitude is a (finite)."""
    if a == 0:
        return 0
    m, k = np.frexp(a)              # 0.5 <= m < 1
    return int(np.clip(k - 1 - (2 if 2 * m <= 1.5 else 1), -126, 127))


def round_e2m1(v: np.ndarray) -> np.ndarray:
    """Codes of the nearest e2m1 values (ties to the even code) of |v| <= 6."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 0, 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(a == MAGNITUDES[hi], hi, pick).astype(np.uint8) | np.where(np.signbit(v), 8, 0).astype(np.uint8)


def pack(x: np.ndarray):
    """(codes [n x f], scale bytes [n x ceil(f / 32)])."""
    x = np.asarray(x, np.float64)
    n, f = x.shape
    nb = -(-f // BLOCK)
    q, s = np.zeros((n, f), np.uint8), np.zeros((n, nb), np.uint8)
    for i in range(n):
        for b in range(nb):
            c = slice(b * BLOCK, min(f, (b + 1) * BLOCK))
            if not np.all(np.isfinite(x[i, c])):
                s[i, b] = 255       # the codes say nothing; zeros
                continue
            e = exponent(float(np.max(np.abs(x[i, c]))))
            q[i, c], s[i, b] = round_e2m1(x[i, c] * 2.0 ** -e), e + 127
    return q, s


def values(q: np.ndarray, s: np.ndarray) -> np.ndarray:
    """What codes under one scale for each 32 columns stand for."""
    e = np.repeat(s.astype(np.float64), BLOCK, 1)[:, :q.shape[1]]
    return np.where(e == 255, np.nan, TABLE[q] * 2.0 ** (np.where(e == 255, 127, e) - 127.0))


def masked(x: np.ndarray, mask) -> np.ndarray:
    return np.asarray(x, np.float64) if mask is None else np.where(np.asarray(mask) > 0, x, 0.0)


def laid_out(q: np.ndarray, s: np.ndarray):
    """Bytes and scales in the library's order, by the formulas of the header, element by element."""
    n, f = q.shape
    P, R = -(-f // 256), -(-n // 64)
    out, sc = np.zeros((n, 128 * P), np.uint8), np.full(512 * P * R, 127, np.uint8)
    for i in range(n):
        for j in range(f):
            out[i, j // 2] |= int(q[i, j]) << (4 * (j % 2))
        for b in range(s.shape[1]):
            sc[512 * ((b // 8) * R + i // 64) + 256 * (b // 4 % 2) + 64 * (b % 4) + 4 * (i % 16) + i // 16 % 4] = s[i, b]
    return out, sc.reshape(P, R, 512)
