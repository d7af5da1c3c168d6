"""Plain NumPy definitions of the orthogonalised update, in float64 (test
infrastructure; the definitions are those of ``include/gcn_muon.h``)."""
from __future__ import annotations

import numpy as np

COEF = (3.4445, -4.7750, 2.0315)
SLOPE = 3.9692     # the largest of the polynomial's slopes on 0 .. 1.2025


def orthogonalise(U, steps: int = 5) -> np.ndarray:
    U = np.asarray(U, np.float64)
    a, b, c = COEF
    if U.shape[0] > U.shape[1]:
        return orthogonalise(U.T, steps).T
    norm = np.sqrt((U * U).sum())
    X = U / norm if norm > 0 else U.copy()
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X


def update(W, G, M, lr, scale, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5):
    """(W, M) after one update."""
    W, G, M = (np.asarray(x, np.float64) for x in (W, G, M))
    M = momentum * M + G
    U = G + momentum * M if nesterov else M
    return (1.0 - lr * weight_decay) * W - lr * scale * orthogonalise(U, steps), M


def error_bound(U, steps: int = 5, unit: float = 2.0 ** -22) -> float:
    """A bound of the 2-norm error of the iteration whose operands are each held within `unit` of their value and
    whose sums of K products are chains of 3 ceil(K / 32) + 4 float32 additions, each within 2^-23 of the sum of
    magnitudes.  What is off in a step's X grows at most SLOPE-fold in the next: the largest slope of the
    polynomial bounds its divided differences, and they the matrix function's."""
    U = np.asarray(U, np.float64)
    if U.shape[0] > U.shape[1]:
        U = U.T
    norm = np.sqrt((U * U).sum())
    if norm == 0:
        return 0.0
    a, b, c = COEF
    fro, two = np.linalg.norm, lambda x: np.linalg.norm(x, 2)

    def sums(p, q):
        return ((3 * -(-p.shape[1] // 32) + 4) * 2.0 ** -23 + 2 * unit) * fro(np.abs(p) @ np.abs(q))

    X = U / norm
    E = 2 * unit
    for _ in range(steps):
        A = X @ X.T
        dA = sums(X, X.T) + unit * fro(A)
        B = b * A + c * (A @ A)
        dB = abs(b) * dA + abs(c) * (2 * two(A) * dA + sums(A, A)) + 4 * unit * (abs(b) * fro(A) + abs(c) * fro(A @ A))
        Xn = a * X + B @ X
        E = SLOPE * E + dB * two(X) + sums(B, X) + 4 * unit * (a * fro(X) + fro(Xn))
        X = Xn
    return float(E)
