"""Plain NumPy definitions of the 8-bit rows and of the many-class loss, in
float64 (test infrastructure; the definitions are those of
``include/gcn_rows8.h`` and ``include/gcn_classes.h``)."""
from __future__ import annotations

import numpy as np

BLOCK = 128


def e4m3_table() -> np.ndarray:
    """The value of each of the 256 e4m3 bytes."""
    b = np.arange(256)
    s, e, m = np.where(b >= 128, -1.0, 1.0), (b >> 3) & 15, b & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    return np.where((b & 127) == 127, np.nan, s * v)


TABLE = e4m3_table()
_POS = TABLE[:127]     # 0 .. 448, ascending


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """Bytes of the nearest e4m3 values (ties to the even byte) of |v| <= 448."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(a == _POS[hi], hi, pick).astype(np.uint8) | np.where(np.signbit(v), 128, 0).astype(np.uint8)


def exponent(a: float) -> int:
    """Scale exponent of a block whose largest finite magnitude is a."""
    if a == 0:
        return 0
    m, k = np.frexp(a)              # 0.5 <= m < 1
    return int(np.clip(k - 1 - (8 if 2 * m <= 1.75 else 7), -126, 127))


def held(x: np.ndarray, e) -> np.ndarray:
    """Bytes of x 2^-e with the two departures from rounding."""
    fin = np.isfinite(x)
    v = np.where(fin, x, 0.0) * 2.0 ** -np.asarray(e, np.float64)
    q = round_e4m3(v)
    tiny = (q & 127 == 0) & (v != 0)
    q = np.where(tiny, (q & 128) | 1, q)
    return np.where(fin, q, 127).astype(np.uint8)


def _largest(x: np.ndarray) -> float:
    return float(np.max(np.where(np.isfinite(x), np.abs(x), 0.0), initial=0.0))


def pack_rows(x: np.ndarray):
    """(bytes [n x f], scale bytes [n x ceil(f / 128)])."""
    x = np.asarray(x, np.float64)
    n, f = x.shape
    nb = -(-f // BLOCK)
    q, s = np.zeros((n, f), np.uint8), np.zeros((n, nb), np.uint8)
    for i in range(n):
        for b in range(nb):
            c = slice(b * BLOCK, min(f, (b + 1) * BLOCK))
            e = exponent(_largest(x[i, c]))
            q[i, c], s[i, b] = held(x[i, c], e), e + 127
    return q, s


def pack_weights(w: np.ndarray):
    w = np.asarray(w, np.float64)
    K, N = w.shape
    q, s = np.zeros((K, N), np.uint8), np.zeros((-(-K // BLOCK), -(-N // BLOCK)), np.uint8)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            r = (slice(i * BLOCK, min(K, (i + 1) * BLOCK)), slice(j * BLOCK, min(N, (j + 1) * BLOCK)))
            e = exponent(_largest(w[r]))
            q[r], s[i, j] = held(w[r], e), e + 127
    return q, s


def values(q: np.ndarray, s: np.ndarray, rows: int = 1) -> np.ndarray:
    """What bytes under one scale for each `rows` x 128 stand for."""
    e = np.repeat(np.repeat(s.astype(np.float64) - 127.0, rows, 0), BLOCK, 1)[:q.shape[0], :q.shape[1]]
    return TABLE[q] * 2.0 ** e


def positive(q: np.ndarray) -> np.ndarray:
    return (q >= 1) & (q <= 126)


def class_loss(H, W, b, labels):
    """(loss, row_loss, dHL, dW, db, G)."""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    n, C = H.shape[0], W.shape[1]
    labels = np.asarray(labels)
    lab = np.nonzero((labels >= 0) & (labels < C))[0]
    rows, G = np.zeros(n), np.zeros((n, C))
    if lab.size:
        X = H[lab] @ W + (0.0 if b is None else np.asarray(b, np.float64))
        top = X.max(1, keepdims=True)
        lse = top + np.log(np.exp(X - top).sum(1, keepdims=True))
        k = np.arange(lab.size)
        rows[lab] = lse[:, 0] - X[k, labels[lab]]
        P = np.exp(X - lse)
        P[k, labels[lab]] -= 1.0
        G[lab] = P / lab.size
    Hz = np.zeros_like(H)
    Hz[lab] = H[lab]
    return rows.sum() / max(1, lab.size), rows, G @ W.T, Hz.T @ G, G.sum(0), G
