"""8-bit rows on the GPU: packing, the 8-bit product and the backward pass that
reads the rows, against plain float64 definitions."""
import numpy as np
import pytest
import torch

from oracle import rows8 as R
from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


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


def bytes_of(r):
    return r.view(torch.uint8).cpu().numpy() if r.dtype == torch.float8_e4m3fn else r.cpu().numpy()


def rows_of(x):
    """Rows8 of a float64 array by the oracle."""
    q, s = R.pack_rows(x)
    out = B.Rows8(*x.shape)
    out.values.copy_(torch.from_numpy(q).cuda().view(torch.float8_e4m3fn))
    out.scale.copy_(torch.from_numpy(s).cuda())
    return out, R.values(q, s), q


def weights_of(w):
    q, s = R.pack_weights(w)
    out = B.Weights8(*w.shape)
    t = torch.from_numpy(q).cuda()
    out.values.copy_(t.view(torch.float8_e4m3fn))
    out.values_t.copy_(t.T.contiguous().view(torch.float8_e4m3fn))
    out.scale.copy_(torch.from_numpy(s).cuda())
    return out, R.values(q, s, R.BLOCK)


def spread(g, n, f):
    """Values of many sizes: rows and columns of unlike scales, some zeros."""
    x = g.normal(size=(n, f)) * np.exp(2 * g.normal(size=(n, 1))) * np.exp(g.normal(size=(1, f)))
    return np.where(g.random((n, f)) < 0.3, 0.0, x)


# ------------------------------------------------------------------- packing
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, f, pad", [(1, 1, 0), (1, 128, 0), (3, 127, 1), (17, 129, 0), (33, 256, 8), (70, 602, 6),
                                       (5, 50, 3), (200, 640, 0)])
def test_pack_is_exact(n, f, pad, dtype):
    t = DT[dtype]
    x = held(spread(gen(n * 1000 + f), n, f), t)
    X = padded(n, f, t, pad)
    X.copy_(to_dev(x, t))
    r = B.gcn_rows8_pack(X, B.Rows8(n, f))
    q, s = R.pack_rows(x)
    assert np.array_equal(bytes_of(r.scale), s)
    assert np.array_equal(bytes_of(r.values), q)
    # the rest of the last block is zero
    whole = torch.as_strided(r.values.view(torch.uint8), (n, r.struct.ldq), (r.struct.ldq, 1))
    assert int(whole[:, f:].max()) == 0 if f % 128 else True
    # and back, exactly
    out = padded(n, f, torch.float32, pad)
    B.gcn_rows8_unpack(r, out)
    assert np.array_equal(out.cpu().numpy().astype(np.float64), R.values(q, s))
    out16 = torch.empty((n, f), dtype=torch.bfloat16, device="cuda")
    B.gcn_rows8_unpack(r, out16)
    assert np.array_equal(out16.to(torch.float64).cpu().numpy(), R.values(q, s))


def test_pack_every_rounding_case():
    """Halfway values between all neighbours, at several scales, and the rest of the departures."""
    mid = (R.TABLE[:126] + R.TABLE[1:127]) / 2
    base = np.concatenate([mid, [448.0, 0.0]])
    x = np.stack([base, -base, base * 2.0 ** -100, base * 2.0 ** 90, np.nextafter(base.astype(np.float32), np.float32(0)),
                  np.full(128, 2.0 ** -149), np.where(np.arange(128) == 5, np.inf, base),
                  np.where(np.arange(128) == 7, np.nan, -base), np.full(128, np.nan), np.full(128, -np.inf),
                  np.full(128, 3.4e38), np.full(128, -0.0), np.where(np.arange(128) == 0, 1e30, 1e-30)])
    r = B.gcn_rows8_pack(to_dev(x), B.Rows8(*x.shape))
    q, s = R.pack_rows(x.astype(np.float32))
    assert np.array_equal(bytes_of(r.scale), s)
    got = bytes_of(r.values)
    nan = (q & 127) == 127
    assert np.array_equal(got[~nan], q[~nan]) and np.all((got[nan] & 127) == 127)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K, N, pad", [(1, 1, 0), (128, 128, 0), (127, 130, 2), (300, 50, 0), (50, 602, 0)])
def test_pack_weights_is_exact(K, N, pad, dtype):
    t = DT[dtype]
    w = held(spread(gen(K + N), K, N), t)
    W = padded(K, N, t, pad)
    W.copy_(to_dev(w, t))
    r = B.gcn_weights8_pack(W, B.Weights8(K, N))
    q, s = R.pack_weights(w)
    assert np.array_equal(bytes_of(r.scale), s)
    assert np.array_equal(bytes_of(r.values), q) and np.array_equal(bytes_of(r.values_t), q.T)
    for v, c in ((r.values, N), (r.values_t, K)):
        whole = torch.as_strided(v.view(torch.uint8), (v.shape[0], v.stride(0)), (v.stride(0), 1))
        assert c % 128 == 0 or int(whole[:, c:].max()) == 0


# ------------------------------------------------------------------- product
def product_bound(x, w, y, dtype, bias):
    """What a sum of K products may be off by, element by element.

    float32 results: products are exact, and each of at most K + 2 additions
    rounds or cuts by 2^-23 of the sum of magnitudes.  bfloat16 results: within
    each group of 8 products the 8-bit instruction cuts terms at 2^-13 of the
    largest one, 7 terms at most, and the result is rounded by 2^-8."""
    K = x.shape[1]
    mag = np.abs(x) @ np.abs(w) + np.abs(bias)
    tol = (K + 2) * 2.0 ** -23 * mag
    if dtype == torch.bfloat16:
        for k in range(0, K, 8):
            tol += 7 * 2.0 ** -13 * np.max(np.abs(x[:, k:k + 8, None]) * np.abs(w[None, k:k + 8, :]), axis=1)
        tol += 2.0 ** -8 * (np.abs(y) + tol)
    return tol + 1e-37


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, K, N, transpose, pad", [
    (1, 1, 1, False, 0), (1, 512, 300, False, 0), (2, 129, 5, True, 1), (16, 128, 128, False, 0),
    (33, 602, 128, False, 4), (130, 50, 257, True, 0), (300, 256, 64, False, 0), (129, 1030, 131, False, 3),
    (257, 384, 260, True, 0), (40, 700, 515, False, 1), (64, 130, 77, True, 0), (70, 8320, 66, False, 0),
    (7, 8320, 20, False, 0)])
def test_product(n, K, N, transpose, pad, dtype):
    t = DT[dtype]
    g = gen(n + 7 * K + 11 * N)
    X8, x, _ = rows_of(spread(g, n, K))
    W8, w = weights_of(spread(g, N, K) if transpose else spread(g, K, N))
    w = w.T if transpose else w
    b = g.normal(size=N).astype(np.float32) * (np.abs(x @ w).mean() + 1e-3)
    ws = B.Workspace()
    for bias, relu in ((None, False), (b, True)):
        Y = padded(n, N, t, pad)
        B.gcn_rows8_product(X8, W8, Y, ws, bias=None if bias is None else to_dev(bias), relu=relu, transpose=transpose)
        bb = 0.0 if bias is None else bias.astype(np.float64)
        y = x @ w + bb
        tol = product_bound(x, w, y, t, bb * np.ones((1, N)))
        y = np.maximum(y, 0) if relu else y
        got = Y.to(torch.float64).cpu().numpy()
        assert np.all(np.abs(got - y) <= tol), float(np.max(np.abs(got - y) / tol))
        if pad:   # what lies beyond the columns is left alone
            assert float(torch.as_strided(Y, (n, N + pad), (N + pad, 1))[:, N:].min()) == 7.0


@pytest.mark.parametrize("n, K, N, transpose", [(3001, 1400, 3500, False), (4000, 1, 3003, True), (4100, 640, 2900, True),
                                                (33, 4000, 20000, False), (2600, 16500, 4200, False),
                                                (3333, 300, 970, False), (5000, 515, 601, True)])
def test_product_of_many_tiles(n, K, N, transpose):
    """Sizes of the large tiles, against float64 on the GPU; the bound of product_bound."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + K)
    x = torch.randn(n, K, generator=g, device="cuda") * torch.exp(torch.randn(n, 1, generator=g, device="cuda"))
    w = torch.randn(*((N, K) if transpose else (K, N)), generator=g, device="cuda") / 64
    b = torch.randn(N, generator=g, device="cuda")
    X8, W8 = B.gcn_rows8_pack(x, B.Rows8(n, K)), B.gcn_weights8_pack(w, B.Weights8(*w.shape))
    xv = B.gcn_rows8_unpack(X8, torch.empty_like(x)).double()
    e = W8.scale.double().repeat_interleave(128, 0)[:w.shape[0]].repeat_interleave(128, 1)[:, :w.shape[1]] - 127
    wv = W8.values.double() * torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), e)
    wv = wv.T.contiguous() if transpose else wv
    y, mag = xv @ wv + b, xv.abs() @ wv.abs() + b.abs()
    ws = B.Workspace()
    for t in (torch.float32, torch.bfloat16):
        Y = torch.full((n, N), 7.0, dtype=t, device="cuda")
        B.gcn_rows8_product(X8, W8, Y, ws, bias=b, relu=False, transpose=transpose)
        tol = (K + 2) * 2.0 ** -23 * mag
        if t == torch.bfloat16:   # (the largest of 8 products is at most their sum)
            tol = tol + 7 * 2.0 ** -13 * mag
            tol = tol + 2.0 ** -8 * (y.abs() + tol)
        assert bool(((Y.double() - y).abs() <= tol).all()), float(((Y.double() - y).abs() / tol).max())
        again = torch.empty_like(Y)
        B.gcn_rows8_product(X8, W8, again, ws, bias=b, relu=False, transpose=transpose)
        assert torch.equal(Y, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_at_the_ends_of_the_scale(dtype):
    """Scales whose product leaves float32, and blocks of very unlike scale in one sum."""
    x = np.zeros((4, 384))
    x[0, :128], x[0, 128:256], x[0, 256:] = 2.0 ** 100, 2.0 ** -100, 1.0
    x[1, :] = 2.0 ** -120
    x[2, 200] = 3.0
    w = np.zeros((384, 32))
    w[:128], w[128:256], w[256:] = 2.0 ** -120, 2.0 ** 101, 0.5
    X8, xv, _ = rows_of(x)
    W8, wv = weights_of(w)
    Y = torch.empty((4, 32), dtype=DT[dtype], device="cuda")
    B.gcn_rows8_product(X8, W8, Y, B.Workspace())
    assert np.array_equal(Y.to(torch.float64).cpu().numpy(), held(xv @ wv, DT[dtype]))


def test_product_keeps_nan_where_it_is():
    g = gen(5)
    x = g.normal(size=(40, 256))
    x[7, 3], x[9, 200] = np.nan, np.inf
    X8, xv, _ = rows_of(x)
    W8, wv = weights_of(g.normal(size=(256, 48)))
    for t in (torch.float32, torch.bfloat16):
        Y = torch.empty((40, 48), dtype=t, device="cuda")
        B.gcn_rows8_product(X8, W8, Y, B.Workspace(), relu=True)
        nan = torch.isnan(Y).cpu().numpy()
        assert nan[7].all() and nan[9].all() and not np.delete(nan, [7, 9], 0).any()


# --------------------------------------------------------------- weight grad
def masked_grad(dy, q):
    z = torch.from_numpy(np.asarray(dy, np.float32)).to(torch.bfloat16).to(torch.float64).numpy()
    return z if q is None else np.where(R.positive(q), z, 0.0)


def check_grad(n, f, N, dtype, mask=True, pad=0, seed=0, ws=None):
    t = DT[dtype]
    g = gen(seed + n + 3 * f + 5 * N)
    X8, x, _ = rows_of(np.maximum(spread(g, n, f), 0))
    Y8, _, yq = rows_of(np.maximum(g.normal(size=(n, N)), 0))
    dy = held(spread(g, n, N) * 1e-3, t)
    dY = padded(n, N, t, pad)
    dY.copy_(to_dev(dy, t))
    dW = torch.full((f, N + pad), 7.0, device="cuda")[:, :N]
    db, dZ8 = torch.empty(N, device="cuda"), B.Rows8(n, N)
    B.gcn_rows8_weight_grad(X8, dY, dW, ws or B.Workspace(), db=db, mask=Y8.values if mask else None, dZ8=dZ8)
    z = masked_grad(dy, yq if mask else None)
    # products are exact; n additions and the join of the split sums
    tol = (n + 70) * 2.0 ** -23 * (np.abs(x).T @ np.abs(z)) + 1e-37
    err = np.abs(dW.cpu().numpy() - x.T @ z)
    assert np.all(err <= tol), float(np.max(err / tol))
    assert np.all(np.abs(db.cpu().numpy() - z.sum(0)) <= (n + 70) * 2.0 ** -24 * np.abs(z).sum(0) + 1e-37)
    q, s = R.pack_rows(z)
    assert np.array_equal(bytes_of(dZ8.values), q) and np.array_equal(bytes_of(dZ8.scale), s)
    if pad:
        assert float(torch.as_strided(dW, (f, N + pad), (N + pad, 1))[:, N:].min()) == 7.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, f, N, mask, pad", [(1, 1, 1, True, 0), (1, 128, 64, True, 0), (15, 50, 41, False, 1),
                                                (64, 128, 128, True, 0), (65, 129, 130, True, 2),
                                                (700, 300, 100, True, 0), (2003, 602, 64, True, 0),
                                                (5000, 256, 260, False, 4)])
def test_weight_grad(n, f, N, mask, pad, dtype):
    check_grad(n, f, N, dtype, mask, pad)


def test_weight_grad_of_a_column_range():
    """The neighbour branch's half of a layer's output as the mask, and its half of dY."""
    g = gen(3)
    n, f, h = 500, 96, 72
    X8, x, _ = rows_of(g.normal(size=(n, f)))
    Y8, _, yq = rows_of(np.maximum(g.normal(size=(n, 2 * h)), 0))
    dy = held(g.normal(size=(n, 2 * h)), torch.float32)
    dY = to_dev(dy)
    dW = torch.empty((f, h), device="cuda")
    B.gcn_rows8_weight_grad(X8, dY[:, h:], dW, B.Workspace(), mask=Y8.values[:, h:])
    z = masked_grad(dy[:, h:], yq[:, h:])
    assert np.all(np.abs(dW.cpu().numpy() - x.T @ z) <= (n + 70) * 2.0 ** -23 * (np.abs(x).T @ np.abs(z)) + 1e-37)


def test_weight_grad_masked_places_reach_nothing():
    """Infinities and NaN in dY under a mask byte that is not positive, and a mask that leaves nothing."""
    g = gen(4)
    n, f, N = 90, 64, 40
    X8, x, _ = rows_of(g.normal(size=(n, f)))
    y = g.normal(size=(n, N))
    y[5] = 0.0
    y[6, 3] = np.nan
    Y8, _, yq = rows_of(y)
    dy = held(g.normal(size=(n, N)), torch.bfloat16)
    clean = masked_grad(dy, yq)
    dirty = np.where(R.positive(yq), dy, np.where(g.random((n, N)) < 0.5, np.nan, np.inf))
    dW, db, dZ8 = torch.empty((f, N), device="cuda"), torch.empty(N, device="cuda"), B.Rows8(n, N)
    B.gcn_rows8_weight_grad(X8, to_dev(dirty, torch.bfloat16), dW, B.Workspace(), db=db, mask=Y8.values, dZ8=dZ8)
    assert np.all(np.abs(dW.cpu().numpy() - x.T @ clean) <= (n + 70) * 2.0 ** -23 * (np.abs(x).T @ np.abs(clean)) + 1e-37)
    assert np.array_equal(bytes_of(dZ8.values), R.pack_rows(clean)[0])
    none = B.Rows8(n, N)
    none.values.view(torch.uint8).zero_()
    B.gcn_rows8_weight_grad(X8, to_dev(dirty, torch.bfloat16), dW, B.Workspace(), db=db, mask=none.values, dZ8=dZ8)
    assert float(dW.abs().max()) == 0.0 and float(db.abs().max()) == 0.0 and int(dZ8.scale.min()) == 127


def test_weight_grad_of_no_rows():
    dW, db = torch.full((12, 9), 5.0, device="cuda"), torch.full((9,), 5.0, device="cuda")
    B.gcn_rows8_weight_grad(B.Rows8(0, 12), torch.empty((0, 9), device="cuda"), dW, B.Workspace(), db=db)
    assert float(dW.abs().max()) == 0.0 and float(db.abs().max()) == 0.0


def test_weight_grad_against_differences():
    """<dW, D> against the change of sum(dZ * (X8 W)) along D, and db against that of the bias."""
    g = gen(8)
    n, f, N = 200, 40, 24
    X8, x, _ = rows_of(g.normal(size=(n, f)))
    dy = held(g.normal(size=(n, N)), torch.bfloat16)
    dW, db = torch.empty((f, N), device="cuda"), torch.empty(N, device="cuda")
    B.gcn_rows8_weight_grad(X8, to_dev(dy, torch.bfloat16), dW, B.Workspace(), db=db)
    D, e = g.normal(size=(f, N)), g.normal(size=N)
    W = g.normal(size=(f, N))
    loss = lambda t: float((dy * (x @ (W + t * D) + t * e)).sum())   # linear: the difference is exact in t
    want = (loss(0.5) - loss(-0.5))
    got = float((dW.cpu().numpy().astype(np.float64) * D).sum() + (db.cpu().numpy().astype(np.float64) * e).sum())
    scale = float((np.abs(x).T @ np.abs(dy) * np.abs(D)).sum() + (np.abs(dy).sum(0) * np.abs(e)).sum())
    assert abs(got - want) <= (n + 70) * 2.0 ** -23 * scale


# ------------------------------------------------- streams, graphs, repeats
def test_repeats_and_other_streams_give_the_same_bits():
    g = gen(11)
    n, f, N = 3001, 200, 136
    X8, _, _ = rows_of(g.normal(size=(n, f)))
    W8, _ = weights_of(g.normal(size=(f, N)))
    dY = to_dev(g.normal(size=(n, N)))
    ref = None
    for stream in (None, torch.cuda.Stream(), None):
        ws = B.Workspace()
        Y, dW, db = torch.empty((n, N), device="cuda"), torch.empty((f, N), device="cuda"), torch.empty(N, device="cuda")
        ws.get(64 << 20)
        torch.cuda.synchronize()
        B.gcn_rows8_product(X8, W8, Y, ws, relu=True, stream=stream)
        B.gcn_rows8_weight_grad(X8, dY, dW, ws, db=db, stream=stream)
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dW, db)]
        ref = ref or got
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_captured_and_replayed():
    g = gen(12)
    n, f, N = 1500, 160, 96
    x = [g.normal(size=(n, f)) for _ in range(3)]
    w = g.normal(size=(f, N))
    dys = [g.normal(size=(n, N)) for _ in range(3)]
    X, dY = to_dev(x[0]), to_dev(dys[0])
    W8, _ = weights_of(w)

    def make():
        return (B.Rows8(n, f), torch.empty((n, N), dtype=torch.bfloat16, device="cuda"), B.Rows8(n, N),
                torch.empty((f, N), device="cuda"), torch.empty(N, device="cuda"), B.Rows8(n, N))

    def step(X8, Y, Y8, dW, db, dZ8, ws):
        B.gcn_rows8_pack(X, X8)
        B.gcn_rows8_product(X8, W8, Y, ws, relu=True)
        B.gcn_rows8_pack(Y, Y8)
        B.gcn_rows8_weight_grad(X8, dY, dW, ws, db=db, mask=Y8.values, dZ8=dZ8)

    bufs, ws = make(), B.Workspace()
    ws.get(64 << 20)
    step(*bufs, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*bufs, ws)
    for i in (1, 2, 0, 1):
        X.copy_(to_dev(x[i]))
        dY.copy_(to_dev(dys[i]))
        graph.replay()
        eager, ws2 = make(), B.Workspace()
        step(*eager, ws2)
        torch.cuda.synchronize()
        for a, b in zip(bufs, eager):
            if isinstance(a, B.Rows8):
                assert np.array_equal(bytes_of(a.values), bytes_of(b.values)) and torch.equal(a.scale, b.scale)
            else:
                assert torch.equal(a, b)


def test_binding_refuses_other_shapes_and_types():
    X8, W8, ws = B.Rows8(8, 64), B.Weights8(64, 32), B.Workspace()
    with pytest.raises(ValueError):
        B.gcn_rows8_product(X8, W8, torch.empty((8, 33), device="cuda"), ws)
    with pytest.raises(TypeError):
        B.gcn_rows8_product(X8, W8, torch.empty((8, 32), device="cuda", dtype=torch.float16), ws)
    with pytest.raises(B.GcnError):
        B.gcn_rows8_product(B.Rows8(8, 60), W8, torch.empty((8, 32), device="cuda"), ws)
    with pytest.raises(TypeError):
        B.gcn_rows8_pack(torch.empty((8, 64)), X8)
    with pytest.raises(ValueError):
        B.gcn_rows8_weight_grad(X8, torch.empty((8, 32), device="cuda"), torch.empty((64, 31), device="cuda"), ws)
    with pytest.raises(TypeError):
        B.Rows8.of(X8.values, X8.scale.to(torch.int32))
