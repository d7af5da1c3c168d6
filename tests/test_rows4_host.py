"""4-bit rows on the CPU: the oracle against plain definitions, the order of
the scales, and the library's refusals (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import rows4 as R
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
def test_e2m1_table_is_the_format():
    for code in range(16):
        e, m = (code >> 1) & 3, code & 1
        v = (1 + m / 2) * 2.0 ** (e - 1) if e else m / 2
        assert R.TABLE[code] == (-v if code & 8 else v)


def test_rounding_is_nearest_even():
    mid = (R.MAGNITUDES[:-1] + R.MAGNITUDES[1:]) / 2
    assert list(mid) == [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    assert list(R.round_e2m1(mid)) == [0, 2, 2, 4, 4, 6, 6]
    assert list(R.round_e2m1(np.nextafter(mid, 0))) == list(range(7))
    assert list(R.round_e2m1(np.nextafter(mid, 9))) == list(range(1, 8))
    assert list(R.round_e2m1(-R.MAGNITUDES)) == list(range(8, 16))


@pytest.mark.parametrize("a", [1.0, 1.5, np.nextafter(1.5, 2), 6.0, 6.5, 8.0, 2.0 ** -149, 2.0 ** -126, 3e38])
def test_scale_keeps_the_largest_value_in_range(a):
    e = R.exponent(a)
    assert a * 2.0 ** -e <= 6.0
    assert e == -126 or a * 2.0 ** -(e - 1) > 6.0                # and is the smallest such power


def test_a_block_that_is_not_finite_stands_for_nan():
    x = np.ones((1, 70))
    x[0, 40] = np.inf
    q, s = R.pack(x)
    v = R.values(q, s)
    assert np.all(v[0, :32] == 1) and np.all(np.isnan(v[0, 32:64])) and np.all(v[0, 64:] == 1)


@pytest.mark.parametrize("n, f", [(1, 1), (64, 256), (65, 257), (130, 40), (20, 1000)])
def test_order_of_the_scales(n, f):
    g = np.random.default_rng(n + f)
    q = g.integers(0, 16, (n, f)).astype(np.uint8)
    s = g.integers(1, 255, (n, -(-f // 32))).astype(np.uint8)
    got = B.rows4_scales(torch.from_numpy(s)).numpy()
    assert np.array_equal(got, R.laid_out(q, s)[1])


# ---------------------------------------------------------------- refusals
def rows4(n=10, f=300, ldq=256, q=0x20000, scale=0x30000):
    return B.gcn_rows4(n, f, ldq, q, scale)


BAD = [(rows4(ldq=255), B.GCN_ESHAPE), (rows4(ldq=240), B.GCN_ESHAPE), (rows4(ldq=264), B.GCN_ESHAPE),
       (rows4(n=-1), B.GCN_ESHAPE), (rows4(f=-1), B.GCN_ESHAPE), (rows4(q=None), B.GCN_EINVAL),
       (rows4(scale=None), B.GCN_EINVAL), (rows4(q=0x20008), B.GCN_EINVAL), (rows4(scale=0x30004), B.GCN_EINVAL),
       (rows4(f=2 ** 31 - 1, ldq=2 ** 31 - 16), B.GCN_EUNSUPPORTED)]


@pytest.mark.parametrize("r, code", BAD)
def test_bad_rows_are_refused_everywhere(L, r, code):
    ref, good = ctypes.byref(r), rows4(f=max(r.f, 0))
    assert L.gcn_rows4_unpack(ref, FAKE, 0, 2 ** 31 - 1, None) == code
    assert L.gcn_rows4_product(ref, ctypes.byref(good), None, 0, FAKE, 0, 300, FAKE, 1 << 40, None) == code
    assert L.gcn_rows4_product(ctypes.byref(good), ref, None, 0, FAKE, 0, 300, FAKE, 1 << 40, None) in (
        code, B.GCN_EUNSUPPORTED)
    n, f = max(r.n, 0), max(r.f, 0)
    assert L.gcn_rows4_pack(FAKE, 0, n, f, 2 ** 31 - 1, None, 0, ref, None, None, None, 0, None) == code
    assert L.gcn_rows4_pack(FAKE, 0, f, n, 2 ** 31 - 1, None, 0, None, ref, None, None, 0, None) == code


def test_pack_argument_errors(L):
    def pack(X=FAKE, ty=0, n=10, f=300, ldx=300, mask=None, ldm=0, out=rows4(), outT=None, cs=None, ws=FAKE, wb=1 << 40):
        return L.gcn_rows4_pack(X, ty, n, f, ldx, mask, ldm, None if out is None else ctypes.byref(out),
                                None if outT is None else ctypes.byref(outT), cs, ws, wb, None)

    assert pack(ty=2) == B.GCN_EINVAL
    assert pack(n=-1) == B.GCN_ESHAPE
    assert pack(ldx=299) == B.GCN_ESHAPE
    assert pack(mask=FAKE, ldm=299) == B.GCN_ESHAPE
    assert pack(X=None) == B.GCN_EINVAL
    assert pack(X=P(0x10002)) == B.GCN_EINVAL
    assert pack(X=P(0x10001), ty=1) == B.GCN_EINVAL
    assert pack(mask=P(0x10002), ldm=300) == B.GCN_EINVAL
    assert pack(cs=P(0x10002)) == B.GCN_EINVAL
    assert pack(out=None) == B.GCN_EINVAL                        # nothing asked for
    assert pack(out=rows4(n=11)) == B.GCN_ESHAPE
    assert pack(out=rows4(f=299)) == B.GCN_ESHAPE
    assert pack(outT=rows4(n=10, f=300)) == B.GCN_ESHAPE         # f x n is wanted
    need = L.gcn_rows4_pack_workspace_bytes(10, 300)
    assert need > 0
    assert pack(cs=FAKE, wb=need - 1) == B.GCN_EWORKSPACE
    assert pack(cs=FAKE, ws=None) == B.GCN_EWORKSPACE
    assert pack(cs=FAKE, ws=P(0x10010)) == B.GCN_EWORKSPACE
    # nothing to do: no launch
    assert pack(X=None, n=0, out=rows4(n=0, q=None, scale=None)) == B.GCN_OK
    assert pack(X=None, f=0, out=rows4(f=0, ldq=0, q=None, scale=None)) == B.GCN_OK
    assert L.gcn_rows4_pack_workspace_bytes(-1, 5) == 0


def test_unpack_argument_errors(L):
    r = rows4()
    assert L.gcn_rows4_unpack(None, FAKE, 0, 300, None) == B.GCN_EINVAL
    assert L.gcn_rows4_unpack(ctypes.byref(r), None, 0, 300, None) == B.GCN_EINVAL
    assert L.gcn_rows4_unpack(ctypes.byref(r), FAKE, 0, 299, None) == B.GCN_ESHAPE
    assert L.gcn_rows4_unpack(ctypes.byref(r), FAKE, 7, 300, None) == B.GCN_EINVAL
    assert L.gcn_rows4_unpack(ctypes.byref(r), P(0x10002), 0, 300, None) == B.GCN_EINVAL
    e = rows4(n=0, q=None, scale=None)
    assert L.gcn_rows4_unpack(ctypes.byref(e), None, 0, 300, None) == B.GCN_OK


def test_product_argument_errors(L):
    def product(a=rows4(), b=rows4(n=70), bias=None, Y=FAKE, ty=0, ldy=70, ws=FAKE, wb=1 << 40):
        return L.gcn_rows4_product(None if a is None else ctypes.byref(a), ctypes.byref(b), bias, 0, Y, ty, ldy, ws, wb,
                                   None)

    assert product(a=None) == B.GCN_EINVAL
    assert product(a=rows4(f=301)) == B.GCN_ESHAPE
    assert product(ldy=69) == B.GCN_ESHAPE
    assert product(ty=3) == B.GCN_EINVAL
    assert product(Y=None) == B.GCN_EINVAL
    assert product(Y=P(0x10002)) == B.GCN_EINVAL
    assert product(bias=P(0x10002)) == B.GCN_EINVAL
    assert product(ws=None) == B.GCN_EWORKSPACE
    assert product(ws=P(0x10010)) == B.GCN_EWORKSPACE
    assert product(a=rows4(n=0, q=None, scale=None), Y=None) == B.GCN_OK
    assert product(b=rows4(n=0, q=None, scale=None), Y=None) == B.GCN_OK
    need = L.gcn_rows4_product_workspace_bytes(512, 512, 65536)  # few tiles, a long sum: partials
    assert need > 4 * 512 * 512
    a = rows4(n=512, f=65536, ldq=32768)
    assert product(a=a, b=a, ldy=512, wb=need - 1) == B.GCN_EWORKSPACE


@pytest.mark.parametrize("M, N", [(0, 50), (50, 0), (0, 0), (0, 1 << 20), (1 << 20, 0)])
@pytest.mark.parametrize("f", [0, 40, 5888, 5889, 6144, 8000, 65536, 1 << 24])
def test_operands_of_no_rows_at_any_length_of_the_sum(L, M, N, f):
    """Nothing to form: no parts, no launch, whatever the sum's length."""
    assert L.gcn_rows4_product_workspace_bytes(M, N, f) == 256
    ldq = 128 * -(-f // 256)

    def rows(n):
        return rows4(n=n, f=f, ldq=ldq, q=0x20000 if n else None, scale=0x30000 if n else None)

    a, b = rows(M), rows(N)
    assert L.gcn_rows4_product(ctypes.byref(a), ctypes.byref(b), None, 0, None, 0, N, FAKE, 256, None) == B.GCN_OK
    assert L.gcn_rows4_product(ctypes.byref(a), ctypes.byref(b), None, 0, None, 1, N, FAKE, 255, None) == B.GCN_EWORKSPACE
