"""4-bit products on every tile shape with what a layer asks of them (bfloat16
results, bias, ReLU, padded rows), and their gradients by differences."""
import numpy as np
import pytest
import torch

from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture()
def ws():
    return B.Workspace()


def packed(x, ws):
    r = B.Rows4(*x.shape)
    B.gcn_rows4_pack(x, ws, out=r)
    return r, B.gcn_rows4_unpack(r, torch.empty(x.shape, device="cuda"))


# (few rows; 64 x 64, 128 x 128 and 256 x 256 tiles, whole and ragged; long sums in parts of 64 x 64 and 128 x 128 tiles)
SIZES = [(1, 4100, 1000), (33, 70, 6500), (64, 700, 300), (2000, 513, 602), (100, 200, 8000), (512, 256, 8000),
         (1024, 510, 65536), (16384, 512, 512), (4100, 4099, 700), (4100, 4099, 1100), (2561, 4096, 2050)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("M, N, K", SIZES)
def test_layers_product(M, N, K, pad, dtype, ws):
    t = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N + K + pad)
    A4, a = packed(torch.randn((M, K), generator=g, device="cuda") * torch.exp(torch.randn((M, 1), generator=g, device="cuda")), ws)
    B4, b = packed(torch.randn((N, K), generator=g, device="cuda"), ws)
    bias = torch.randn(N, generator=g, device="cuda") * K ** 0.5
    want = a.double() @ b.double().T + bias.double()
    # every instruction adds 128 products to a float32 sum, parts and the bias come after it: each of these additions is
    # off by at most two half steps of the magnitudes so far
    tol = (-(-K // 128) + 66) * 2.0 ** -22 * (a.double().abs() @ b.double().abs().T + bias.double().abs())
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    for relu in (True, False):
        Y = torch.full((M, N + pad), 7.0, dtype=t, device="cuda")[:, :N]
        B.gcn_rows4_product(A4, B4, Y, ws, bias=bias, relu=relu)
        off = (Y.double() - (want.clamp(min=0) if relu else want)).abs()
        assert bool((off <= tol).all())
        if relu:
            assert bool((Y >= 0).all())
        if pad:
            assert bool((Y.as_strided((M, pad), (N + pad, 1), N) == 7.0).all())


def grid(shape, g):
    """Values that 4 bits hold under the scale one, with a 4 or a 6 in every 32 of a row and of a column: both
    orientations hold them exactly."""
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    x = v[torch.randint(0, 8, shape, generator=g)] * (torch.randint(0, 2, shape, generator=g) * 2 - 1)
    i, j = torch.arange(shape[0])[:, None], torch.arange(shape[1])[None]
    return torch.where((i + j) % 16 == 0, 4.0, x)


@pytest.mark.parametrize("n, K, N", [(70, 40, 33), (40, 300, 20), (700, 130, 260), (300, 64, 1030)])
def test_gradients_are_differences_of_the_product(n, K, N, ws):
    """L = <X4 W4, dZ>: L's differences for a step of one weight, or of one input, between values that its block holds
    are that element of dW = X4^T dZ4, or of dX = dZ4 W4^T.  Everything is halves below 2^21: exact in float32."""
    g = torch.Generator().manual_seed(n + K)
    x, w, dz = grid((n, K), g), grid((K, N), g), grid((n, N), g)

    def both(v):
        r, t = B.Rows4(*v.shape), B.Rows4(*v.T.shape)
        B.gcn_rows4_pack(v.cuda(), ws, out=r, out_t=t)
        for p, q in ((r, v), (t, v.T)):
            assert torch.equal(B.gcn_rows4_unpack(p, torch.empty(q.shape, device="cuda")).cpu(), q)
        return r, t

    def total(x4, w4t):
        Y = B.gcn_rows4_product(x4, w4t, torch.empty((n, N), device="cuda"), ws)
        return float((Y.double().cpu() * dz.double()).sum())

    (X4, X4T), (W4, W4T), (Z4, Z4T) = both(x), both(w), both(dz)
    dX = B.gcn_rows4_product(Z4, W4, torch.empty((n, K), device="cuda"), ws).cpu()
    dW = B.gcn_rows4_product(X4T, Z4T, torch.empty((K, N), device="cuda"), ws).cpu()
    rng = np.random.default_rng(n)
    for v, d, at in ((w, dW, 0), (x, dX, 1)):
        small = torch.nonzero(v.abs() <= 1.0)                # (half a step up and down is held, too)
        for i, j in small[torch.from_numpy(rng.choice(len(small), 12, replace=False))].tolist():
            L = []
            for h in (0.5, -0.5):
                moved = v.clone()
                moved[i, j] += h
                r, t = both(moved)
                L.append(total(X4, t) if at == 0 else total(r, W4T))
            assert L[0] - L[1] == float(d[i, j]), (at, i, j)
