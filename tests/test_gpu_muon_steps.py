"""The orthogonalised update over many steps: directions far below the norm,
which every step brings up 3.4445-fold, against float64."""
import numpy as np
import pytest
import torch

from oracle import muon as O
from tests.gpu_util import require_gpu
from tests.test_gpu_muon import f32_iteration, to_dev
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu
A, B_, C = O.COEF


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture()
def ws():
    return B.Workspace()


def polynomial(x):
    return A * x + B_ * x ** 3 + C * x ** 5


def growth(lo, hi):
    """How much a difference of two rows of 2-norms lo .. hi grows in a step: along the rows at most by the largest |p'|
    (at the ends or where p'' is zero), across them by the largest p(x) / x (at the ends)."""
    at = np.stack([lo, hi] + [np.clip(v, lo, hi) for v in (0.0, np.sqrt(-3 * B_ / (10 * C)))])
    return np.maximum(np.abs(A + 3 * B_ * at ** 2 + 5 * C * at ** 4), np.abs(A + B_ * at ** 2 + C * at ** 4)).max(0)


def apart(sizes, per, rng):
    """Rows of these 2-norms with `per` columns each that no other row has: they stay apart in every product, and a
    row's 2-norm goes through the polynomial alone."""
    u = np.zeros((len(sizes), len(sizes) * per), np.float32)
    for i, s in enumerate(sizes):
        v = rng.uniform(0.5, 1.0, per) * rng.choice([-1.0, 1.0], per)
        u[i, i * per:(i + 1) * per] = s * v / np.linalg.norm(v)
    return u


def bound_apart(x, steps, last, per, rounded):
    """How far a row of `per` elements is off: its square sum e and the factor a + b e + c e^2 are a few float32
    operations, each within 2^-24 of the terms: 2^-21 of them.  Between the steps its elements are float32, from the
    `last` ones on within 2^-22 of themselves or 2^-40 of the norm.  rounded: e is there that of a row rounded to float16,
    2^-10 off."""
    def held(x, left):
        return 2.0 ** -21 * x + np.sqrt(per) * 2.0 ** -40 if left <= last else 2.0 ** -23 * x

    E = held(x, steps)
    for left in range(steps, 0, -1):
        y = np.minimum(x + E, 1.21)
        E = growth(np.maximum(x - E, 0), y) * E + 2.0 ** -21 * y * (A - B_ * y ** 2 + C * y ** 4)
        E += (rounded and left <= last) * 2.0 ** -10 * y * (-B_ * y ** 2 + 2 * C * y ** 4)
        x = polynomial(x)
        E = np.minimum(E + held(x, left - 1), 2.5)   # (no two rows within 1.21 are further apart)
    return E


SHAPES = [(3, 2, False), (60, 2, True), (40, 60, False), (100, 5, False), (300, 2, True), (600, 2, False), (1100, 1, False)]


@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
@pytest.mark.parametrize("steps", [5, 6, 7, 8, 9, 12, 13, 14, 15, 20, 30, 64])
@pytest.mark.parametrize("rows, per, tall", SHAPES)
def test_rows_apart(rows, per, tall, steps, prec, ws):
    """Sizes from 1 to what the last step brings to about one; float32 ahead of the last 6 steps (GCN_BF16: 12)."""
    u = apart(np.logspace(0, -0.5371 * steps, rows), per, np.random.default_rng(rows + steps))
    w = np.linalg.norm(u.astype(np.float64), axis=1)
    x = w / np.linalg.norm(w)
    want = x.copy()
    for _ in range(steps):
        want = polynomial(want)
    tol = bound_apart(x, steps, 6 if prec == B.GCN_F32 else 12, per, prec == B.GCN_BF16 and rows >= 128)
    v = to_dev(u.T if tall else u)
    got = B.gcn_orthogonalise(v, torch.empty_like(v), ws, steps=steps, prec=prec).double().cpu().numpy()
    got = got.T if tall else got
    off = np.linalg.norm(got - u.astype(np.float64) * (want / w)[:, None], axis=1)
    far = off > tol + 2.0 ** -23 * want
    assert not far.any(), (np.flatnonzero(far)[:5], off[far][:5], tol[far][:5])


@pytest.mark.parametrize("rows, cols", [(40, 60), (20, 3000), (100, 300), (300, 130), (400, 700), (900, 1000)])
@pytest.mark.parametrize("steps, size", [(6, 6e-4), (7, 2e-4), (8, 1e-4), (9, 2e-5), (13, 1e-6), (20, 1e-10), (30, 1e-13)])
def test_rows_of_unlike_sizes(rows, cols, steps, size, ws):
    """Half of the rows so much smaller: they come out right by themselves, as near as four times float32 products'."""
    g = np.random.default_rng(rows + steps)
    u = g.normal(size=(rows, cols)).astype(np.float32)
    small = np.arange(rows) % 2 == 1
    if rows > cols:   # (few columns: their sizes)
        small = np.arange(cols) % 2 == 1
        u[:, small] *= np.float32(size)
    else:
        u[small] *= np.float32(size)
    want, plain = O.orthogonalise(u, steps), f32_iteration(u, steps)
    v = to_dev(u)
    got = B.gcn_orthogonalise(v, torch.empty_like(v), ws, steps=steps).double().cpu().numpy()
    for part in (small, ~small):
        of = (lambda a: a[:, part]) if rows > cols else (lambda a: a[part])   # noqa: E731
        norm = np.linalg.norm(of(want))
        err, base = np.linalg.norm(of(got - want)) / norm, np.linalg.norm(of(plain - want)) / norm
        assert err <= 4 * base + 2.0 ** -21, (err, base)


@pytest.mark.parametrize("rows, cols, gt", [(40, 60, torch.float32), (700, 300, torch.bfloat16), (130, 2000, torch.float32)])
def test_updates_of_many_steps(rows, cols, gt, ws):
    """The momentum, the decay and W's padding as in updates of few steps."""
    g = np.random.default_rng(rows)
    W = torch.full((rows, cols + 3), 7.0, device="cuda")[:, :cols]
    w, m = g.normal(size=(rows, cols)).astype(np.float32), g.normal(size=(rows, cols)).astype(np.float32)
    G = to_dev(g.normal(size=(rows, cols)), gt)
    M = to_dev(m)
    W.copy_(to_dev(w))
    gr = G.double().cpu().numpy()
    B.MuonStep([W], [G], [M], scales=[2.0], weight_decay=0.1, steps=9)(0.02, ws)
    want, wm = O.update(w, gr, m, 0.02, 2.0, weight_decay=0.1, steps=9)
    u = gr + 0.95 * wm
    o, p = O.orthogonalise(u, 9), f32_iteration(u, 9)
    assert np.all(np.abs(M.cpu().numpy() - wm) <= 2.0 ** -23 * (np.abs(m) + np.abs(gr)))
    tol = 4 * np.linalg.norm(p - o) + 2.0 ** -20 * np.linalg.norm(o)
    assert np.linalg.norm(W.cpu().numpy() - want) <= 0.04 * tol + 2.0 ** -22 * np.linalg.norm(w)
    assert bool((W.as_strided((rows, 3), (cols + 3, 1), cols) == 7.0).all())


def test_captured_update_of_many_steps():
    """Replayed between eager updates of the same matrices."""
    g = np.random.default_rng(3)
    W, G, M = (to_dev(g.normal(size=(200, 150))) for _ in range(3))
    w, m = W.clone(), M.clone()
    ws, other = B.Workspace(), B.Workspace()
    ws.get(1 << 24)
    step, eager = B.MuonStep([W], [G], [M], steps=10), B.MuonStep([w], [G], [m], steps=10)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(0.05, ws)
    for _ in range(4):
        graph.replay()
        eager(0.05, other)
        torch.cuda.synchronize()
        assert torch.equal(W, w) and torch.equal(M, m)


@pytest.mark.parametrize("rows, cols", [(1500, 1500), (2300, 1030), (2050, 2300), (2500, 2500), (3000, 3300)])
def test_large_sides_of_many_steps(rows, cols, ws):
    """The other tile shapes, against the iteration in float64 on the GPU; a third of the rows far smaller."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    u = torch.randn((rows, cols), generator=g, device="cuda")
    (u.T if rows > cols else u)[::3] *= 2.0 ** -13
    out = torch.empty_like(u)
    for prec, steps in ((B.GCN_F32, 8), (B.GCN_BF16, 13)):
        B.gcn_orthogonalise(u, out, ws, steps=steps, prec=prec)
        x = u.double() / u.double().norm()
        x = x.T.contiguous() if rows > cols else x
        y = x.float()
        for _ in range(steps):
            s = x @ x.T
            x = A * x + (B_ * s + C * (s @ s)) @ x
            s = y @ y.T
            y = A * y + (B_ * s + C * (s @ s)) @ y
        x, y = (x.T, y.T) if rows > cols else (x, y)
        err, plain = (float((v.double() - x).norm() / x.norm()) for v in (out, y))
        # (GCN_BF16: twelve steps in float16, each within 2^-9; a step carries that on by -1.58 at the fixed point 0.868, by
        # 1.2 around the cycle 0.70, 1.11: 1.45 taken.  A lost part or a wrong index is off by about one.)
        assert err <= (4 * plain + 2.0 ** -21 if prec == B.GCN_F32 else 2.0 ** -9 * sum(1.45 ** k for k in range(12))), prec


@pytest.mark.parametrize("rows, cols", [(40, 70), (300, 200)])
@pytest.mark.parametrize("prec, steps", [(B.GCN_F32, 7), (B.GCN_BF16, 13), (B.GCN_F32, 64)])
def test_zeros_and_values_that_are_not_finite(rows, cols, prec, steps, ws):
    x = torch.zeros((rows, cols), device="cuda")
    out = torch.full_like(x, 5.0)
    B.gcn_orthogonalise(x, out, ws, steps=steps, prec=prec)
    assert not out.any()
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.randn((rows, cols), device="cuda")
        x[7, 9] = bad
        B.gcn_orthogonalise(x, out, ws, steps=steps, prec=prec)
        assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("rows, cols", [(70, 90), (300, 200)])
def test_scale_does_not_matter(rows, cols, ws):
    """A power of two changes no bit; the matrix may be its own result; bfloat16 results are float32's, rounded."""
    x = torch.randn((rows, cols), generator=torch.Generator().manual_seed(rows)).bfloat16().float().cuda()
    base = B.gcn_orthogonalise(x, torch.empty_like(x), ws, steps=10)
    for k in (-100, -20, 60, 120):
        assert torch.equal(B.gcn_orthogonalise(x * 2.0 ** k, torch.empty_like(x), ws, steps=10), base), k
    half = x.bfloat16()
    assert torch.equal(B.gcn_orthogonalise(half, half, ws, steps=10), base.bfloat16())
    assert torch.equal(B.gcn_orthogonalise(x, x, ws, steps=10), base)


@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("prec, steps", [(B.GCN_F32, 2), (B.GCN_BF16, 2), (B.GCN_F32, 7)])
def test_matrices_past_32_bit_offsets(prec, steps, tall, ws):
    """More than 2^31 elements, one in each row: what every row comes to is known, and everything else is zero."""
    rows, cols = 36_000, 60_000
    i = torch.arange(rows, device="cuda")
    at = i * 5 // 3
    s = torch.logspace(0, -2, rows, dtype=torch.float64, device="cuda")[i * 7 % rows].float()
    u = torch.zeros((cols, rows) if tall else (rows, cols), device="cuda")
    place = (at, i) if tall else (i, at)
    u[place] = s
    out = torch.full_like(u, 5.0)
    B.gcn_orthogonalise(u, out, ws, steps=steps, prec=prec)
    x = s.double() / s.double().norm()
    for _ in range(steps):
        x = polynomial(x)
    # A step's few roundings of 2^-22 (float16's of e, 2^-10 of a term below 2^-9 of the factor, x being below 0.02 at the
    # start): below 2^-20, and not larger in the next, where |x p'(x) / p(x)| < 1 up to 0.7.  Beyond, which more than
    # three steps reach, it is below 5: three such steps 2^7
    assert float(((out[place].double() - x) / x).abs().max()) < 2.0 ** (-17 if steps == 2 else -13)
    out[place] = 0.0
    assert not out.any()
