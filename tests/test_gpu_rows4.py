"""4-bit rows on the GPU: packing in both orientations, reading back, and the
product, against plain float64 definitions."""
import numpy as np
import pytest
import torch

from oracle import rows4 as R
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


def gen(seed):
    return np.random.default_rng(seed)


def to_dev(x, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda").to(dtype)


def held(x, dtype):
    """x as the array type holds it, in float64."""
    return torch.from_numpy(np.asarray(x, np.float32)).to(dtype).to(torch.float64).numpy()


def padded(n, f, dtype, pad):
    """An n x f view of rows pad elements longer."""
    return torch.full((n, f + pad), 7.0, dtype=dtype, device="cuda")[:, :f]


def spread(g, n, f):
    """Values of many sizes: rows and columns of unlike scales, some zeros."""
    x = g.normal(size=(n, f)) * np.exp(2 * g.normal(size=(n, 1))) * np.exp(g.normal(size=(1, f)))
    return np.where(g.random((n, f)) < 0.3, 0.0, x)


def rows_of(x):
    """Rows4 of a float64 array by the oracle, and what they stand for."""
    q, s = R.pack(x)
    v, sc = R.laid_out(q, s)
    return B.Rows4.of(torch.from_numpy(v).cuda(), torch.from_numpy(sc).cuda(), x.shape[1]), R.values(q, s)


def check_rows(r, x):
    """r holds the 4-bit rows of x, zeros behind the last column, nothing behind the last row."""
    n, f = x.shape
    q, s = R.pack(x)
    v, sc = R.laid_out(q, s)
    assert np.array_equal(r.values.cpu().numpy(), v)
    got = r.scale.cpu().numpy()
    P, G = got.shape[:2]
    k = np.arange(512)
    row = k // 4 % 16 + 16 * (k % 4) + 64 * np.arange(G)[:, None]          # [G, 512]
    assert np.array_equal(got[:, row < n], sc[:, row < n])
    assert not got[:, row >= n].any()                                       # as they were allocated


# ------------------------------------------------------------------- packing
SHAPES = [(1, 1, 0), (1, 256, 0), (3, 31, 1), (17, 33, 0), (33, 255, 8), (65, 257, 3), (129, 50, 5), (300, 128, 0),
          (64, 602, 6), (128, 64, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, f, pad", SHAPES)
def test_pack_is_exact(n, f, pad, dtype, ws):
    t = DT[dtype]
    g = gen(n * 1000 + f)
    x = held(spread(g, n, f), t)
    m = held(g.normal(size=(n, f)), t)
    X, M = padded(n, f, t, pad), padded(n, f, t, 2 * pad)
    X.copy_(to_dev(x, t))
    M.copy_(to_dev(m, t))
    for mask in (None, M):
        z = R.masked(x, None if mask is None else m)
        only, out, out_t = B.Rows4(n, f), B.Rows4(n, f), B.Rows4(f, n)
        cs = torch.empty(f, device="cuda")
        B.gcn_rows4_pack(X, ws, out=only, mask=mask)
        check_rows(only, z)
        B.gcn_rows4_pack(X, ws, out=out, out_t=out_t, mask=mask, colsum=cs)
        check_rows(out, z)
        check_rows(out_t, z.T)
        # n - 1 additions, each rounded by at most 2^-24 of what is summed so far
        assert np.all(np.abs(cs.cpu().numpy() - z.sum(0)) <= n * 2.0 ** -24 * np.abs(z).sum(0) + 1e-300)
        other, alone = B.Rows4(f, n), torch.empty(f, device="cuda")
        B.gcn_rows4_pack(X, ws, out_t=other, mask=mask)
        B.gcn_rows4_pack(X, ws, colsum=alone, mask=mask)
        assert torch.equal(other.values, out_t.values) and torch.equal(other.scale, out_t.scale)
        assert torch.equal(alone, cs)
        # and back, exactly
        q, s = R.pack(z)
        v = padded(n, f, torch.float32, pad)
        B.gcn_rows4_unpack(out, v)
        assert np.array_equal(v.cpu().numpy().astype(np.float64), R.values(q, s))
        v16 = torch.empty((n, f), dtype=torch.bfloat16, device="cuda")
        B.gcn_rows4_unpack(out, v16)
        assert np.array_equal(v16.to(torch.float64).cpu().numpy(), R.values(q, s))
        if pad:   # nothing behind the rows
            assert bool((v.as_strided((n, pad), (f + pad, 1), f) == 7.0).all())


def test_pack_every_rounding_case(ws):
    """Halfway values between all neighbours and their neighbours, at several scales, and what is not finite."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    base = np.zeros(32)
    base[:7], base[7] = mid, 6.0
    base[8:15], base[15:22] = np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(9))
    base[22:30] = R.MAGNITUDES
    x = np.stack([base, -base, base * 2.0 ** -100, base * 2.0 ** -126, base * 2.0 ** -140, base * 2.0 ** 124,
                  np.full(32, 2.0 ** -149), np.where(np.arange(32) == 5, np.inf, base),
                  np.where(np.arange(32) == 31, np.nan, -base), np.full(32, np.nan), np.full(32, -np.inf),
                  np.full(32, 3.4e38), np.full(32, -0.0), np.where(np.arange(32) == 0, 1e30, 1e-30),
                  np.full(32, 1.5), np.nextafter(np.full(32, 1.5, np.float32), np.float32(2)), np.zeros(32)])
    x = x.astype(np.float32).astype(np.float64)
    r, t = B.Rows4(*x.shape), B.Rows4(*x.T.shape)
    B.gcn_rows4_pack(to_dev(x), ws, out=r, out_t=t)
    check_rows(r, x)
    check_rows(t, x.T)
    v = torch.empty(x.shape, device="cuda")
    B.gcn_rows4_unpack(r, v)
    with np.errstate(over="ignore"):   # (3.4e38 is held as 4 * 2^126, which float32 does not hold: infinity)
        want = R.values(*R.pack(x)).astype(np.float32)
    assert np.array_equal(v.cpu().numpy(), want, equal_nan=True)
    # under a mask what is not finite there does not count
    m = np.where(np.isfinite(x), 1.0, 0.0)
    B.gcn_rows4_pack(to_dev(x), ws, out=r, out_t=t, mask=to_dev(m))
    check_rows(r, R.masked(x, m))
    check_rows(t, R.masked(x, m).T)


def test_unpack_every_code_under_every_scale():
    q = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    s = np.arange(256, dtype=np.uint8)[:, None]
    v, sc = R.laid_out(q, s)
    out = torch.empty((256, 32), device="cuda")
    B.gcn_rows4_unpack(B.Rows4.of(torch.from_numpy(v).cuda(), torch.from_numpy(sc).cuda(), 32), out)
    with np.errstate(over="ignore"):
        want = R.values(q, s).astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)


def test_mask_values():
    """Zero, negative zero, NaN and negative infinity are not positive; the smallest subnormal is."""
    m = torch.tensor([[0.0, -0.0, float("nan"), float("-inf"), 2.0 ** -149, float("inf"), 1.0, -1.0]], device="cuda")
    x = torch.full((1, 8), 2.0, device="cuda")
    r, v = B.Rows4(1, 8), torch.empty((1, 8), device="cuda")
    B.gcn_rows4_pack(x, B.Workspace(), out=r, mask=m)
    B.gcn_rows4_unpack(r, v)
    assert v.tolist() == [[0, 0, 0, 0, 2, 2, 2, 0]]


def test_no_rows(ws):
    X = torch.empty((0, 40), device="cuda")
    cs = torch.full((40,), 3.0, device="cuda")
    out, out_t = B.Rows4(0, 40), B.Rows4(40, 0)
    B.gcn_rows4_pack(X, ws, out=out, out_t=out_t, colsum=cs)
    assert not cs.any()
    # a sum over nothing: the bias alone
    Y = torch.empty((40, 40), device="cuda")
    b = torch.linspace(-1, 1, 40, device="cuda")
    B.gcn_rows4_product(out_t, out_t, Y, ws, bias=b, relu=True)
    assert torch.equal(Y, torch.relu(b).expand(40, 40))
    assert B.gcn_rows4_product(out, out, torch.empty((0, 0), device="cuda"), ws).numel() == 0


@pytest.mark.parametrize("M, N", [(100, 70), (2600, 2700)])
def test_sums_over_nothing(M, N, ws):
    """Tiles without a piece."""
    b = torch.linspace(-1, 1, N, device="cuda")
    Y = torch.empty((M, N), device="cuda")
    B.gcn_rows4_product(B.Rows4(M, 0), B.Rows4(N, 0), Y, ws, bias=b)
    assert torch.equal(Y, b.expand(M, N))


# ------------------------------------------------------------------- product
def sum_bound(K, a, b):
    """Every instruction adds 128 products to a float32 sum, parts and the bias are added after it: each of these
    additions is off by at most two half steps of what is summed so far."""
    return (-(-K // 128) + 66) * 2.0 ** -22 * (np.abs(a) @ np.abs(b).T)


PRODUCTS = [(1, 1, 1), (1, 300, 4096), (5, 17, 33), (16, 16, 256), (17, 100, 257), (33, 64, 602), (64, 130, 512),
            (65, 63, 50), (100, 200, 2050), (257, 129, 96), (300, 1000, 700), (130, 70, 5000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M, N, K", PRODUCTS)
def test_product(M, N, K, dtype, ws):
    t = DT[dtype]
    g = gen(M + 3 * N + 7 * K)
    A4, a = rows_of(spread(g, M, K))
    B4, b = rows_of(g.normal(size=(N, K)))
    bias = g.normal(size=N).astype(np.float32)
    for relu, use in ((False, False), (True, True)):
        Y = padded(M, N, t, 3)
        B.gcn_rows4_product(A4, B4, Y, ws, bias=to_dev(bias) if use else None, relu=relu)
        want = a @ b.T + (bias.astype(np.float64) if use else 0.0)
        tol = sum_bound(K, a, b) + 2.0 ** -23 * np.abs(want)
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
        want = np.maximum(want, 0.0) if relu else want
        assert np.all(np.abs(Y.to(torch.float64).cpu().numpy() - want) <= tol)
        assert bool((Y.as_strided((M, 3), (N + 3, 1), N) == 7.0).all())     # nothing behind the rows


def test_product_of_whole_numbers_is_exact(ws):
    """Small whole numbers: every sum below 2^24 is exact in any order, on every tile shape."""
    for M, N, K in ((40, 500, 1024), (300, 300, 512), (1500, 1600, 640), (4100, 4096, 1024), (600, 520, 40000),
                    (50, 130, 30000), (200, 130, 6500), (1024, 512, 65536)):
        g = torch.Generator(device="cuda")
        g.manual_seed(M)
        x = torch.randint(-3, 4, (M, K), generator=g, device="cuda").float()
        y = torch.randint(-3, 4, (N, K), generator=g, device="cuda").float()
        x[:, ::32], y[:, ::32] = 4.0, 4.0      # (every block's scale is one)
        A4, B4 = B.Rows4(M, K), B.Rows4(N, K)
        B.gcn_rows4_pack(x, ws, out=A4)
        B.gcn_rows4_pack(y, ws, out=B4)
        Y = torch.empty((M, N), device="cuda")
        B.gcn_rows4_product(A4, B4, Y, ws)
        assert torch.equal(Y, x @ y.T), (M, N, K)


def test_scales_differ_from_block_to_block(ws):
    """Every block of both operands under another scale: a byte taken from the wrong row or block shows."""
    for M, N, K in ((64, 64, 512), (200, 200, 1024), (3400, 3000, 1100)):
        g = gen(M)
        a = np.ones((M, K)) * 2.0 ** np.repeat(g.integers(-6, 7, (M, -(-K // 32))), 32, 1)[:, :K]
        b = np.ones((N, K)) * 2.0 ** np.repeat(g.integers(-6, 7, (N, -(-K // 32))), 32, 1)[:, :K]
        A4, B4 = B.Rows4(M, K), B.Rows4(N, K)
        B.gcn_rows4_pack(to_dev(a), ws, out=A4)
        B.gcn_rows4_pack(to_dev(b), ws, out=B4)
        Y = torch.empty((M, N), device="cuda")
        B.gcn_rows4_product(A4, B4, Y, ws)
        want = a @ b.T                          # multiples of 2^-12 below 2^23: within a few steps of float32
        assert np.abs(Y.cpu().numpy() / want - 1).max() < 2.0 ** -20


@pytest.mark.parametrize("M, N, K", [(8, 40, 300), (200, 150, 600), (3400, 3000, 1024)])
def test_nan_reaches_its_row_and_column_alone(M, N, K, ws):
    g = gen(5)
    a, b = g.normal(size=(M, K)), g.normal(size=(N, K))
    a[M // 2, K - 1] = np.inf
    b[N - 1, 0] = np.nan
    A4, B4 = B.Rows4(M, K), B.Rows4(N, K)
    B.gcn_rows4_pack(to_dev(a), ws, out=A4)
    B.gcn_rows4_pack(to_dev(b), ws, out=B4)
    Y = torch.empty((M, N), device="cuda")
    B.gcn_rows4_product(A4, B4, Y, ws, relu=True)
    want = np.zeros((M, N), bool)
    want[M // 2], want[:, N - 1] = True, True
    assert np.array_equal(np.isnan(Y.cpu().numpy()), want)


def test_products_are_the_layers_gradients(ws):
    """Y = X4 W4, and with dZ: dX = dZ4 W4^T and dW = X4^T dZ4 are the gradients of <Y, dZ> in the packed values,
    each by its own orientation's blocks; against differences of the product itself."""
    n, K, N = 70, 40, 33
    g = gen(1)
    x, w, dy, y = (held(g.normal(size=s), torch.float32) for s in ((n, K), (K, N), (n, N), (n, N)))
    X4, X4T, W4, W4T = B.Rows4(n, K), B.Rows4(K, n), B.Rows4(K, N), B.Rows4(N, K)
    dZ4, dZ4T, db = B.Rows4(n, N), B.Rows4(N, n), torch.empty(N, device="cuda")
    B.gcn_rows4_pack(to_dev(x), ws, out=X4, out_t=X4T)
    B.gcn_rows4_pack(to_dev(w), ws, out=W4, out_t=W4T)
    B.gcn_rows4_pack(to_dev(dy), ws, out=dZ4, out_t=dZ4T, mask=to_dev(y), colsum=db)
    Y, dX, dW = (torch.empty(s, device="cuda") for s in ((n, N), (n, K), (K, N)))
    B.gcn_rows4_product(X4, W4T, Y, ws)
    B.gcn_rows4_product(dZ4, W4, dX, ws)
    B.gcn_rows4_product(X4T, dZ4T, dW, ws)
    V = lambda a: R.values(*R.pack(a))                                                     # noqa: E731
    z = R.masked(dy, y)
    for got, a, b, k in ((Y, V(x), V(w.T), K), (dX, V(z), V(w), N), (dW, V(x.T), V(z.T), n)):
        assert np.all(np.abs(got.cpu().numpy() - a @ b.T) <= sum_bound(k, a, b))
    # a step of one weight that its block holds exactly moves <Y, dZ> by that weight's gradient
    v = V(w.T).T
    for k, j in ((0, 0), (7, 32), (39, 5)):
        h = 2.0 ** -6
        up, dn = v.copy(), v.copy()
        up[k, j] += h
        dn[k, j] -= h
        diff = ((V(x) @ up) * V(z)).sum() - ((V(x) @ dn) * V(z)).sum()
        assert abs(diff / (2 * h) - V(x)[:, k] @ V(z)[:, j]) < 1e-9


def test_another_stream_and_a_captured_graph():
    """The calls follow the current stream, and replay from a graph with eager work between the replays."""
    g = gen(9)
    x, w, dy = (to_dev(g.normal(size=s)) for s in ((300, 200), (150, 200), (300, 9000)))
    ws = B.Workspace()

    def run(ws):
        X4, W4, D4T = B.Rows4(300, 200), B.Rows4(150, 200), B.Rows4(9000, 300)
        X4T, Y, dW, cs = B.Rows4(200, 300), torch.empty((300, 150), device="cuda"), None, torch.empty(9000, device="cuda")
        B.gcn_rows4_pack(x, ws, out=X4, out_t=X4T)
        B.gcn_rows4_pack(w, ws, out=W4)
        B.gcn_rows4_pack(dy, ws, out_t=D4T, mask=dy, colsum=cs)
        B.gcn_rows4_product(X4, W4, Y, ws, relu=True)
        L4, M4 = B.Rows4(200, 9000), B.Rows4(120, 9000)      # a long sum in parts
        B.gcn_rows4_pack(dy[:200], ws, out=L4)
        B.gcn_rows4_pack(dy[100:220], ws, out=M4)
        dW = torch.empty((200, 120), device="cuda")
        B.gcn_rows4_product(L4, M4, dW, ws)
        v = torch.empty((9000, 300), device="cuda", dtype=torch.bfloat16)
        B.gcn_rows4_unpack(D4T, v)
        return Y, cs, dW, v

    want = [t.clone() for t in run(ws)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run(B.Workspace())
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws2 = B.Workspace()
    ws2.get(1 << 24)
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = run(ws2)
    for _ in range(4):
        for t in got:
            t.zero_()
        graph.replay()
        eager = run(ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, e) for a, b, e in zip(got, want, eager))


def test_rows_past_32_bit_offsets(ws):
    """More than 2^31 elements, in both orientations: the last rows as packed alone, and a sum over all of them."""
    n, f, tail = 2_100_032, 1056, 320                         # (n - tail a multiple of 64: whole groups and blocks)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    X = torch.empty((n, f), dtype=torch.bfloat16, device="cuda")
    part = torch.randn((4096, f), generator=g, device="cuda")
    for i in range(0, n, 4096):
        m = min(4096, n - i)
        X[i:i + m] = part[:m] * 2.0 ** (i // 4096 % 7 - 3)
    out, out_t = B.Rows4(n, f), B.Rows4(f, n)
    B.gcn_rows4_pack(X, ws, out=out, out_t=out_t)
    last, last_t = B.Rows4(tail, f), B.Rows4(f, tail)
    B.gcn_rows4_pack(X[n - tail:], ws, out=last, out_t=last_t)
    assert torch.equal(out.values[n - tail:], last.values)
    assert torch.equal(out.scale[:, (n - tail) // 64:], last.scale)
    assert torch.equal(out_t.values[:, (n - tail) // 2:n // 2], last_t.values[:, :tail // 2])
    v, w = torch.empty((n, f), dtype=torch.bfloat16, device="cuda"), torch.empty((tail, f), device="cuda")
    B.gcn_rows4_unpack(out, v)
    B.gcn_rows4_unpack(last, w)
    assert torch.equal(v[n - tail:].float(), w)
    # X^T X over all rows is the sum of two parts' (whole pieces of 256 each)
    del v
    half = n // 512 * 256
    Y = torch.empty((f, f), device="cuda")
    B.gcn_rows4_product(out_t, out_t, Y, ws)
    sums = torch.zeros((f, f), dtype=torch.float64, device="cuda")
    for a, b in ((0, half), (half, n)):
        p = B.Rows4.of(out_t.values[:, a // 2:], out_t.scale[a // 256:-(-b // 256)], b - a) if b == n else \
            B.Rows4.of(out_t.values[:, a // 2:b // 2], out_t.scale[a // 256:b // 256], b - a)
        y = torch.empty((f, f), device="cuda")
        B.gcn_rows4_product(p, p, y, ws)
        sums += y.double()
    # each is a float32 sum: within sqrt(K / 128) half steps of its size in the 2-norm, and all three far below this
    assert float((Y.double() - sums).norm() / sums.norm()) < 128 * 2.0 ** -24
