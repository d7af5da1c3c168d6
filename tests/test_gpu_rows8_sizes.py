"""8-bit rows at the sizes whose kernels and launch shapes small ones do not
reach: 17 to 32 rows of the product, packing beyond one grid, the weight
gradient of large tiles and strips of many rows."""
import numpy as np
import pytest
import torch

from oracle import rows8 as R
from tests.gpu_util import require_gpu
from tests import test_gpu_rows8 as small
from tests.test_gpu_rows8 import DT, bytes_of, gen, product_bound, rows_of, spread, to_dev, weights_of
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, K, N, transpose", [(17, 300, 70, False), (32, 1100, 33, True), (31, 4096, 130, False),
                                                (48, 260, 40, False), (64, 640, 1, True), (65, 640, 17, False)])
def test_product_of_few_rows(n, K, N, transpose, dtype):
    g = gen(n * 31 + K)
    X8, x, _ = rows_of(spread(g, n, K))
    W8, w = weights_of(spread(g, N, K) if transpose else spread(g, K, N))
    w = w.T if transpose else w
    b = g.normal(size=N).astype(np.float32)
    Y = torch.full((n, N + 3), 7.0, dtype=DT[dtype], device="cuda")
    B.gcn_rows8_product(X8, W8, Y[:, :N], B.Workspace(), bias=to_dev(b), relu=False, transpose=transpose)
    y = x @ w + b.astype(np.float64)
    tol = product_bound(x, w, y, DT[dtype], b.astype(np.float64) * np.ones((1, N)))
    err = np.abs(Y[:, :N].to(torch.float64).cpu().numpy() - y)
    assert np.all(err <= tol), float(np.max(err / tol))
    assert float(Y[:, N:].min()) == 7.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_beyond_one_grid(dtype):
    """350,000 blocks and 5.25 million pieces of eight: bytes of sampled rows against the definition, every value
    against what half a step allows."""
    n, f = 70000, 600
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    x = (torch.randn(n, f, generator=g, device="cuda") * torch.exp(torch.randn(n, 1, generator=g, device="cuda"))).to(DT[dtype])
    r = B.gcn_rows8_pack(x, B.Rows8(n, f))
    some = np.r_[0:3, 1000:n:1500, 52428:52431, n - 3:n]   # (row 52,428 ends the first sweep of the grid)
    q, s = R.pack_rows(x[some].to(torch.float64).cpu().numpy())
    assert np.array_equal(bytes_of(r.values[some]), q) and np.array_equal(bytes_of(r.scale[some]), s)
    v = B.gcn_rows8_unpack(r, torch.full((n, f), 7.0, device="cuda")).double()
    scale = torch.exp2(r.scale.double() - 127).repeat_interleave(128, 1)[:, :f]
    assert bool(((v - x.double()).abs() <= 2.0 ** -4 * x.double().abs() + 2.0 ** -9 * scale).all())
    assert np.array_equal(v[some].cpu().numpy(), R.values(q, s))


@pytest.mark.parametrize("n, f, N, dtype, mask", [(40003, 1000, 500, "bf16", True), (40003, 1000, 500, "f32", True),
                                                  (65536, 1024, 512, "bf16", True), (50021, 131, 260, "f32", False),
                                                  (65536, 602, 64, "bf16", True), (33000, 2000, 777, "f32", True)])
def test_weight_grad_of_large_subgraphs(n, f, N, dtype, mask):
    g = torch.Generator(device="cuda")
    g.manual_seed(n + f)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    X8 = B.gcn_rows8_pack(torch.relu(normal(n, f)), B.Rows8(n, f))
    Y8 = B.gcn_rows8_pack(torch.relu(normal(n, N)), B.Rows8(n, N))
    dY = (normal(n, N) * 1e-3 * torch.exp(normal(n, 1))).to(DT[dtype])
    dW, db, dZ8 = torch.full((f, N), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), B.Rows8(n, N)
    B.gcn_rows8_weight_grad(X8, dY, dW, B.Workspace(), db=db, mask=Y8.values if mask else None, dZ8=dZ8)
    x = X8.values.double() * torch.exp2(X8.scale.double() - 127).repeat_interleave(128, 1)[:, :f]
    z = dY.to(torch.bfloat16).double()
    if mask:
        z = torch.where(Y8.values.float() > 0, z, 0.0)
    # products are exact; n additions and the join of the split sums
    want, mag = x.T.contiguous() @ z, x.abs().T.contiguous() @ z.abs()
    err = (dW.double() - want).abs()
    assert bool((err <= (n + 70) * 2.0 ** -23 * mag + 1e-37).all())
    # (errors of random signs: far below that bound; a product that missed a row of n would be 1 / sqrt(n) off)
    assert float(err.norm()) <= 2.0 ** -18 * float(want.norm())
    assert bool(((db.double() - z.sum(0)).abs() <= (n + 70) * 2.0 ** -24 * z.abs().sum(0) + 1e-37).all())
    some = np.r_[0:20, 77:n:701, n - 20:n]
    q, s = R.pack_rows(z[some].cpu().numpy())
    assert np.array_equal(bytes_of(dZ8.values[some]), q) and np.array_equal(bytes_of(dZ8.scale[some]), s)
    v = B.gcn_rows8_unpack(dZ8, torch.empty((n, N), device="cuda")).double()
    scale = torch.exp2(dZ8.scale.double() - 127).repeat_interleave(128, 1)[:, :N]
    assert bool(((v - z).abs() <= 2.0 ** -4 * z.abs() + 2.0 ** -9 * scale).all())


@pytest.mark.parametrize("n, K, N, transpose", [(6400, 700, 500, False), (6145, 300, 1000, True), (12288, 129, 512, False),
                                                (12300, 260, 512, False), (6400, 4096, 512, False)])
def test_product_about_the_edges_of_a_tile_size(n, K, N, transpose):
    """From 384 to 768 tiles of 64 x 128, and one row of tiles more."""
    small.test_product_of_many_tiles(n, K, N, transpose)


@pytest.mark.parametrize("shift", [-149, -140, -134, -127, -118, 120])
def test_pack_and_unpack_at_the_ends_of_the_types(shift):
    """Blocks from float32's smallest subnormal to its largest values: bytes, scales and what comes back, in float32
    exactly and in bfloat16 rounded once."""
    g = gen(shift + 1000)
    x = np.ldexp(g.integers(-15, 16, size=(6, 300)).astype(np.float64), shift)
    x[0, :128], x[1, 5], x[2, 7] = 0.0, -0.0, np.ldexp(1.0, -149)
    r = B.gcn_rows8_pack(to_dev(x), B.Rows8(6, 300))
    q, s = R.pack_rows(x)
    assert np.array_equal(bytes_of(r.values), q) and np.array_equal(bytes_of(r.scale), s)
    v = R.values(q, s)
    out = B.gcn_rows8_unpack(r, torch.empty((6, 300), device="cuda"))
    assert np.array_equal(out.cpu().numpy().astype(np.float64), v)
    out = B.gcn_rows8_unpack(r, torch.empty((6, 300), dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(out.cpu(), torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16))
