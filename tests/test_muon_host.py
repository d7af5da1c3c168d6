"""The orthogonalised update on the CPU: the oracle against the singular value
decomposition, and the library's refusals (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest

from oracle import muon as O
from paper_1810_11899_amd import binding as B
from paper_1810_11899_amd import build as pkg_build

P = ctypes.c_void_p
FAKE = P(0x10000)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pkg_build.LIB_PATH):
        pkg_build.build_library()
    return B.lib()


@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 9), (9, 1), (12, 30), (30, 12), (20, 20)])
def test_oracle_maps_the_singular_values(rows, cols):
    U = np.random.default_rng(rows * 50 + cols).normal(size=(rows, cols))
    l, s, r = np.linalg.svd(U, full_matrices=False)
    x = s / np.sqrt((s ** 2).sum())
    for _ in range(5):
        x = O.COEF[0] * x + O.COEF[1] * x ** 3 + O.COEF[2] * x ** 5
    assert np.abs(O.orthogonalise(U) - (l * x) @ r).max() < 1e-12


def test_polynomial_stays_in_its_bounds():
    """0 .. 1.2025 goes into itself, A's eigenvalues stay below 1.446 and B's within -2.807 .. 0: what the scaled float16
    operands are laid out for."""
    a, b, c = O.COEF
    x = np.linspace(0, 1.2025, 200001)
    y = a * x + b * x ** 3 + c * x ** 5
    assert y.min() >= 0 and y.max() <= 1.2025
    lam = x * x
    assert lam.max() < 1.4461 and (b * lam + c * lam ** 2).min() > -2.807 and (b * lam + c * lam ** 2).max() <= 0
    assert np.abs(a + 3 * b * x ** 2 + 5 * c * x ** 4).max() <= O.SLOPE    # at the upper end; 3.4445 at zero
    assert 1.2025 * 2 ** 15 < 65504 and 1.4461 * 2 ** 14 < 65504 and 2.807 * 2 ** 13 < 65504


def test_update_oracle_is_its_formula():
    g = np.random.default_rng(0)
    W, G, M = (g.normal(size=(5, 8)) for _ in range(3))
    w, m = O.update(W, G, M, 0.1, 2.0, momentum=0.5, nesterov=True, weight_decay=0.25)
    assert np.allclose(m, 0.5 * M + G, rtol=1e-15)
    assert np.allclose(w, (1 - 0.025) * W - 0.2 * O.orthogonalise(G + 0.5 * m), rtol=1e-14)
    w, _ = O.update(W, G, M, 0.1, 2.0, momentum=0.5, nesterov=False)
    assert np.allclose(w, W - 0.2 * O.orthogonalise(m), rtol=1e-14)


# ---------------------------------------------------------------- refusals
def test_orthogonalise_argument_errors(L):
    def call(X=FAKE, ty=0, rows=10, cols=20, ldx=20, out=P(0x90000), ldo=20, steps=5, prec=0, ws=FAKE, wb=1 << 40):
        return L.gcn_orthogonalise(X, ty, rows, cols, ldx, out, ldo, steps, prec, ws, wb, None)

    assert call(ty=2) == B.GCN_EINVAL
    assert call(prec=2) == B.GCN_EINVAL
    assert call(steps=0) == B.GCN_EINVAL
    assert call(steps=65) == B.GCN_EINVAL
    assert call(rows=-1) == B.GCN_ESHAPE
    assert call(ldx=19) == B.GCN_ESHAPE
    assert call(ldo=19) == B.GCN_ESHAPE
    assert call(X=None) == B.GCN_EINVAL
    assert call(out=None) == B.GCN_EINVAL
    assert call(X=P(0x10002)) == B.GCN_EINVAL
    assert call(out=P(0x90001), ty=1) == B.GCN_EINVAL
    assert call(rows=65537) == B.GCN_EUNSUPPORTED
    assert call(cols=65537, ldx=65537, ldo=65537) == B.GCN_EUNSUPPORTED
    assert call(ws=None) == B.GCN_EWORKSPACE
    assert call(ws=P(0x10010)) == B.GCN_EWORKSPACE
    need = L.gcn_orthogonalise_workspace_bytes(10, 20, 0)
    assert need > 0 and call(wb=need - 1) == B.GCN_EWORKSPACE
    assert call(out=P(0x10004)) == B.GCN_EINVAL                  # overlaps X
    assert call(out=FAKE, ldo=24) == B.GCN_EINVAL                # X itself, other rows
    assert call(X=None, out=None, rows=0) == B.GCN_OK
    assert call(X=None, out=None, cols=0, ldx=0, ldo=0) == B.GCN_OK
    assert L.gcn_orthogonalise_workspace_bytes(-1, 5, 0) == 0
    assert L.gcn_orthogonalise_workspace_bytes(5, 5, 3) == 0


def mat(rows=10, cols=20, ldw=20, ldg=20, ldm=20, W=0x10000, G=0x20000, M=0x30000, scale=1.0):
    return B.gcn_muon_matrix(rows, cols, ldw, ldg, ldm, W, G, M, scale)


def update(L, mats, ty=0, lr=0.1, mu=0.9, wd=0.0, steps=5, prec=0, ws=P(0x40000000), wb=1 << 40, count=None):
    arr = (B.gcn_muon_matrix * max(1, len(mats)))(*mats)
    return L.gcn_muon_update(len(mats) if count is None else count, arr if mats else None, ty, lr, mu, 1, wd, steps, prec, ws,
                             wb, None)


def test_update_argument_errors(L):
    def one(code, match="", **kw):
        m = {k: kw.pop(k) for k in list(kw) if k in ("rows", "cols", "ldw", "ldg", "ldm", "W", "G", "M", "scale")}
        assert update(L, [mat(rows=3, W=0x50000, G=0x60000, M=0x70000), mat(**m)], **kw) == code
        assert match in L.gcn_last_error().decode()

    one(B.GCN_EINVAL, ty=2)
    one(B.GCN_EINVAL, prec=-1)
    one(B.GCN_EINVAL, steps=0)
    one(B.GCN_EINVAL, lr=float("nan"))
    one(B.GCN_EINVAL, mu=1.0)
    one(B.GCN_EINVAL, mu=-0.1)
    one(B.GCN_EINVAL, wd=float("inf"))
    one(B.GCN_EINVAL, scale=float("nan"), match="matrix 1")
    one(B.GCN_ESHAPE, rows=-1)
    one(B.GCN_ESHAPE, ldw=19, match="matrix 1")
    one(B.GCN_ESHAPE, ldg=19)
    one(B.GCN_ESHAPE, ldm=19)
    one(B.GCN_EUNSUPPORTED, rows=65537)
    for x in ("W", "G", "M"):
        one(B.GCN_EINVAL, **{x: None})
        one(B.GCN_EINVAL, **{x: 0x10002})
    one(B.GCN_EWORKSPACE, ws=None)
    one(B.GCN_EWORKSPACE, ws=P(0x10010))
    arr = (B.gcn_muon_matrix * 1)(mat())
    need = L.gcn_muon_workspace_bytes(1, arr, 0)
    assert need > 0 and update(L, [mat()], wb=need - 1) == B.GCN_EWORKSPACE
    assert update(L, [], count=-1) == B.GCN_EINVAL
    assert update(L, [], count=1) == B.GCN_EINVAL
    assert update(L, []) == B.GCN_OK                             # nothing to do: no launch
    assert update(L, [mat(rows=0, W=None, G=None, M=None)]) == B.GCN_OK
    assert update(L, [mat(cols=0, ldw=0, ldg=0, ldm=0)]) == B.GCN_OK


def test_overlaps_are_refused_and_neighbours_are_not(L):
    """Past the overlap check the workspace is too small, which says that the matrices were accepted."""
    far = dict(W=0x500000, G=0x600000, M=0x700000)

    def both(a, b):
        return update(L, [a, b], wb=0)

    assert both(mat(), mat(**far)) == B.GCN_EWORKSPACE
    assert both(mat(), mat(**dict(far, W=0x10000))) == B.GCN_EINVAL            # the same weights twice
    assert both(mat(), mat(**dict(far, M=0x30000))) == B.GCN_EINVAL
    assert both(mat(), mat(**dict(far, W=0x10000 + 799))) == B.GCN_EINVAL      # (misaligned, too)
    assert both(mat(), mat(**dict(far, W=0x10000 + 796))) == B.GCN_EINVAL      # the last element
    assert both(mat(), mat(**dict(far, W=0x10000 + 800))) == B.GCN_EWORKSPACE  # right behind it
    assert both(mat(), mat(**dict(far, W=0x20000))) == B.GCN_EINVAL            # another's gradient
    assert both(mat(), mat(**dict(far, G=0x20000))) == B.GCN_EWORKSPACE        # one gradient for two: read only
    assert both(mat(W=0x30000), mat(**far)) == B.GCN_EINVAL                    # a matrix's own W and M
    # column ranges of one array, side by side
    a, b = mat(ldw=40), mat(**dict(far, W=0x10000 + 80), ldw=40)
    assert both(a, b) == B.GCN_EWORKSPACE and both(b, a) == B.GCN_EWORKSPACE
    assert both(a, mat(**dict(far, W=0x10000 + 76), ldw=40)) == B.GCN_EINVAL
    assert both(a, mat(**dict(far, W=0x10000 + 84), ldw=40)) == B.GCN_EINVAL   # its end runs into the next row
