"""8-bit rows and the many-class loss on the CPU: the oracle against plain
definitions and differences, and the library's refusals (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest

from oracle import rows8 as R
from paper_1810_11899_amd import binding as B
from paper_1810_11899_amd import build as pkg_build

P = ctypes.c_void_p
FAKE = P(0x10000)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pkg_build.LIB_PATH):
        pkg_build.build_library()
    return B.lib()


# ------------------------------------------------------------------ oracle
def test_e4m3_table():
    t = R.TABLE
    assert t[0x7E] == 448.0 and t[1] == 2.0 ** -9 and t[0x38] == 1.0 and np.isnan(t[0x7F]) and np.isnan(t[0xFF])
    assert np.all(np.diff(t[:127]) > 0) and np.array_equal(t[128:255], -t[:127])


def test_rounding_is_nearest_even():
    t = R.TABLE[:127]
    mid = (t[:-1] + t[1:]) / 2
    q = R.round_e4m3(mid)
    assert np.all(q % 2 == 0)                                    # ties to the even byte
    assert np.array_equal(R.round_e4m3(np.nextafter(mid, 0)), np.arange(126))
    assert np.array_equal(R.round_e4m3(np.nextafter(mid, 1e9)), np.arange(1, 127))
    assert np.array_equal(R.round_e4m3(-t), np.arange(127) | 128)


@pytest.mark.parametrize("a", [1.0, 1.75, np.nextafter(1.75, 2), 448.0, 449.0, 2.0 ** -149, 2.0 ** -126, 3e38])
def test_scale_keeps_the_largest_value_in_range(a):
    e = R.exponent(a)
    assert a * 2.0 ** -e <= 448.0
    assert e == -126 or a * 2.0 ** -(e - 1) > 448.0              # and is the smallest such power


def test_a_value_keeps_its_sign():
    x = np.array([[1e6, 1e-9, -1e-9, 0.0, -0.0, np.inf, np.nan]])
    q, s = R.pack_rows(x)
    assert list(q[0, 1:]) == [1, 0x81, 0, 0x80, 0x7F, 0x7F] and s[0, 0] == R.exponent(1e6) + 127


def test_loss_oracle_against_differences():
    g = np.random.default_rng(0)
    n, f, C = 5, 7, 11
    H, W, b = g.normal(size=(n, f)), g.normal(size=(f, C)), g.normal(size=C)
    lab = np.array([3, -1, 10, 0, 11])
    _, _, dH, dW, db, _ = R.class_loss(H, W, b, lab)
    h = 1e-6

    def diff(at, x):
        d = np.zeros_like(x)
        for i in np.ndindex(*x.shape):
            keep = x[i]
            x[i] = keep + h
            up = R.class_loss(H, W, b, lab)[0]
            x[i] = keep - h
            d[i] = (up - R.class_loss(H, W, b, lab)[0]) / (2 * h)
            x[i] = keep
        return d

    # central differences: h^2 of the third derivative and 2^-52 / h of rounding
    for got, x in ((dH, H), (dW, W), (db, b)):
        assert np.abs(got - diff(None, x)).max() < 1e-8


# ---------------------------------------------------------------- refusals
def rows8(n=10, f=200, ldq=256, lds=2, q=0x20000, scale=0x30000):
    return B.gcn_rows8(n, f, ldq, lds, q, scale)


def weights8(K=200, N=300, ldq=384, ldqT=256, lds=3, q=0x40000, qT=0x50000, scale=0x60000):
    return B.gcn_weights8(K, N, ldq, ldqT, lds, q, qT, scale)


@pytest.mark.parametrize("r, code", [
    (rows8(ldq=255), B.GCN_ESHAPE), (rows8(ldq=240), B.GCN_ESHAPE), (rows8(ldq=264), B.GCN_ESHAPE),
    (rows8(lds=1), B.GCN_ESHAPE), (rows8(n=-1), B.GCN_ESHAPE), (rows8(f=0), B.GCN_ESHAPE),
    (rows8(q=None), B.GCN_EINVAL), (rows8(scale=None), B.GCN_EINVAL), (rows8(q=0x20008), B.GCN_EINVAL)])
def test_bad_rows8_are_refused_everywhere(L, r, code):
    w = weights8()
    assert L.gcn_rows8_pack(FAKE, 0, 200, ctypes.byref(r), None) == code
    assert L.gcn_rows8_unpack(ctypes.byref(r), FAKE, 0, 200, None) == code
    assert L.gcn_rows8_product(ctypes.byref(r), ctypes.byref(w), 0, None, 0, FAKE, 0, 300, FAKE, 1 << 40, None) == code
    assert L.gcn_rows8_weight_grad(ctypes.byref(r), None, 0, FAKE, 0, 64, 64, FAKE, 64, None, None, FAKE, 1 << 40,
                                   None) == code


def test_pack_argument_errors(L):
    r = rows8()
    assert L.gcn_rows8_pack(FAKE, 2, 200, ctypes.byref(r), None) == B.GCN_EINVAL
    assert L.gcn_rows8_pack(FAKE, 0, 199, ctypes.byref(r), None) == B.GCN_ESHAPE
    assert L.gcn_rows8_pack(None, 0, 200, ctypes.byref(r), None) == B.GCN_EINVAL
    assert L.gcn_rows8_pack(P(0x10002), 0, 200, ctypes.byref(r), None) == B.GCN_EINVAL
    assert L.gcn_rows8_pack(P(0x10001), 1, 200, ctypes.byref(r), None) == B.GCN_EINVAL
    assert L.gcn_rows8_pack(FAKE, 0, 200, None, None) == B.GCN_EINVAL
    assert L.gcn_rows8_unpack(ctypes.byref(r), None, 1, 200, None) == B.GCN_EINVAL
    assert L.gcn_rows8_unpack(ctypes.byref(r), FAKE, 1, 100, None) == B.GCN_ESHAPE
    empty = rows8(n=0, q=None, scale=None)
    assert L.gcn_rows8_pack(None, 0, 200, ctypes.byref(empty), None) == B.GCN_OK


@pytest.mark.parametrize("w, ldw, code", [
    (weights8(), 299, B.GCN_ESHAPE), (weights8(K=0), 300, B.GCN_ESHAPE), (weights8(ldq=368), 300, B.GCN_ESHAPE),
    (weights8(ldqT=250), 300, B.GCN_ESHAPE), (weights8(lds=2), 300, B.GCN_ESHAPE),
    (weights8(q=None, qT=None), 300, B.GCN_EINVAL), (weights8(scale=None), 300, B.GCN_EINVAL)])
def test_weights_argument_errors(L, w, ldw, code):
    assert L.gcn_weights8_pack(FAKE, 0, ldw, ctypes.byref(w), None) == code


def test_product_argument_errors(L):
    def product(r=rows8(), w=weights8(), t=0, Y=FAKE, ty=0, ldy=300, ws=FAKE, wb=1 << 40):
        return L.gcn_rows8_product(ctypes.byref(r), ctypes.byref(w), t, None, 0, Y, ty, ldy, ws, wb, None)

    assert product(ldy=299) == B.GCN_ESHAPE
    assert product(ty=3) == B.GCN_EINVAL
    assert product(Y=None) == B.GCN_EINVAL
    assert product(ws=None) == B.GCN_EWORKSPACE
    assert product(wb=0) == B.GCN_EWORKSPACE
    assert product(t=1, ldy=300) == B.GCN_ESHAPE                 # X8 has 200 columns, W8^T contracts 300
    assert product(w=weights8(K=201)) == B.GCN_ESHAPE
    assert product(w=weights8(qT=None)) == B.GCN_EINVAL
    assert "orientation" in L.gcn_last_error().decode()
    assert product(r=rows8(f=300, ldq=384, lds=3), w=weights8(q=None), t=1) == B.GCN_EINVAL
    assert product(w=weights8(ldqT=240)) == B.GCN_ESHAPE
    assert product(r=rows8(n=0, q=None, scale=None), Y=None) == B.GCN_OK
    assert product(Y=P(0x10002)) == B.GCN_EINVAL                 # float32 at a 2-byte address
    assert product(ws=P(0x10010)) == B.GCN_EWORKSPACE
    need = L.gcn_rows8_product_workspace_bytes(500, 4096, 512)   # few tiles, long sums: partials
    assert need > 4 * 500 * 512
    r, w = rows8(n=500, f=4096, ldq=4096, lds=32), weights8(K=4096, N=512, ldq=512, ldqT=4096, lds=4)
    assert L.gcn_rows8_product(ctypes.byref(r), ctypes.byref(w), 0, None, 0, FAKE, 0, 512, FAKE, need - 1,
                               None) == B.GCN_EWORKSPACE


def test_weight_grad_argument_errors(L):
    def wg(mask=None, ldm=0, dY=FAKE, ty=0, lddy=64, N=64, dW=FAKE, lddw=64, dz=None, ws=FAKE, wb=1 << 40):
        r = rows8()
        return L.gcn_rows8_weight_grad(ctypes.byref(r), mask, ldm, dY, ty, lddy, N, dW, lddw, None,
                                       None if dz is None else ctypes.byref(dz), ws, wb, None)

    assert wg(N=0) == B.GCN_ESHAPE
    assert wg(lddy=63) == B.GCN_ESHAPE
    assert wg(lddw=63) == B.GCN_ESHAPE
    assert wg(mask=FAKE, ldm=63) == B.GCN_ESHAPE
    assert wg(ty=-1) == B.GCN_EINVAL
    assert wg(dW=None) == B.GCN_EINVAL
    assert wg(dY=None) == B.GCN_EINVAL
    assert wg(dY=P(0x10002)) == B.GCN_EINVAL
    assert wg(dW=P(0x10002)) == B.GCN_EINVAL
    assert wg(dz=rows8(f=63)) == B.GCN_ESHAPE
    assert wg(dz=rows8(n=9, f=64)) == B.GCN_ESHAPE
    assert wg(wb=L.gcn_rows8_weight_grad_workspace_bytes(10, 200, 64) - 1) == B.GCN_EWORKSPACE
    assert wg(ws=P(0x10010)) == B.GCN_EWORKSPACE


def test_class_loss_argument_errors(L):
    def loss(n=10, f=8, ld=8, C=5, H=FAKE, W=FAKE, labels=FAKE, ty=0, out=FAKE, dH=FAKE, ldd=8, dW=FAKE, db=FAKE,
             ws=FAKE, wb=1 << 40):
        return L.gcn_class_loss(H, n, f, ld, W, None, C, labels, ty, out, None, dH, ldd, dW, db, ws, wb, None)

    assert loss(ld=7) == B.GCN_ESHAPE
    assert loss(ldd=7) == B.GCN_ESHAPE
    assert loss(n=-1) == B.GCN_ESHAPE
    assert loss(C=0) == B.GCN_ESHAPE
    assert loss(ty=2) == B.GCN_EINVAL
    for missing in ("H", "W", "labels", "out", "dH", "dW", "db"):
        assert loss(**{missing: None}) == B.GCN_EINVAL, missing
    assert loss(dH=None, db=None) == B.GCN_EINVAL
    assert loss(H=P(0x10002)) == B.GCN_EINVAL                     # float32 at a 2-byte address
    assert loss(wb=8) == B.GCN_EWORKSPACE
    assert loss(ws=P(0x10010)) == B.GCN_EWORKSPACE
    need = L.gcn_class_loss_workspace_bytes(10, 8, 5, 0, 1)
    assert need > 0 and loss(wb=need - 1) == B.GCN_EWORKSPACE
    assert loss(C=2 ** 31 - 1) == B.GCN_EUNSUPPORTED


@pytest.mark.parametrize("n, f, C", [(1, 1, 1), (16384, 1024, 131072), (1 << 20, 512, 200000), (0, 64, 10)])
def test_class_loss_workspace_stays_below_the_logits(L, n, f, C):
    """The query grows with the operands and one piece, not with n x C."""
    for ty, el in ((0, 4), (1, 2)):
        need = L.gcn_class_loss_workspace_bytes(n, f, C, ty, 1)
        operands = 4 * (n * f + f * min(C, 1 << 16)) * 40
        assert 0 < need < operands + (5 << 30)
        assert L.gcn_class_loss_workspace_bytes(n, f, C, ty, 0) <= need
