"""The orthogonalised update on the GPU against plain float64 definitions."""
import numpy as np
import pytest
import torch

from oracle import muon as O
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


def rel2(got, want):
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / n if n else np.linalg.norm(got)


def f32_iteration(U, steps=5):
    """The same iteration in float32 products, for how far off such products are."""
    U = np.asarray(U, np.float64)
    if U.shape[0] > U.shape[1]:
        return f32_iteration(U.T, steps).T
    n = np.linalg.norm(U)
    X = (U / n if n else U).astype(np.float32)
    a, b, c = (np.float32(v) for v in O.COEF)
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.astype(np.float64)


def gradient(g, rows, cols, n=500):
    """As a layer forms it: activations after a ReLU against gradients of unlike rows."""
    return np.maximum(g.normal(size=(rows, n)) + 0.3, 0) @ (g.normal(size=(n, cols)) * np.exp(g.normal(size=(n, 1)))) * 1e-3


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 3), (31, 33), (33, 31), (50, 64), (64, 64), (65, 65), (602, 128), (128, 130), (300, 256),
          (257, 1000), (1000, 40), (64, 2000), (2000, 33), (20, 2081), (1, 6000), (8200, 17)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_orthogonalise(rows, cols, dtype, ws):
    t = DT[dtype]
    g = gen(rows * 7 + cols)
    u = held(gradient(g, rows, cols), t)
    X, out = padded(rows, cols, t, 3), padded(rows, cols, t, 5)
    X.copy_(to_dev(u, t))
    want = O.orthogonalise(u)
    half = torch.finfo(t).eps / 2
    B.gcn_orthogonalise(X, out, ws)
    got = out.to(torch.float64).cpu().numpy()
    # the bound of the arithmetic, and as near as four times float32 products' own error
    norm = np.linalg.norm(want)
    assert np.linalg.norm(got - want) <= O.error_bound(u) + half * norm
    assert rel2(got, want) <= 4 * rel2(f32_iteration(u), want) + 2.0 ** -21 + half
    assert bool((out.as_strided((rows, 5), (cols + 5, 1), cols) == 7.0).all())
    assert torch.equal(X.to(torch.float64).cpu(), torch.from_numpy(u))
    # Operands within 2^-12 (root mean square 2^-11 / sqrt 3): four rounded operands a step (X twice, A, B), weighted by
    # |b| |A|, |c| |A|^2, |B| |X| of about one and not amplified (a X is not rounded): below 2^-9 a step, and
    # of the steps before the last only what the polynomial's slopes of -1.6 .. 1.3 there leave: within 2^-8
    B.gcn_orthogonalise(X, out, ws, prec=B.GCN_BF16)
    assert rel2(out.to(torch.float64).cpu().numpy(), want) <= 2.0 ** -8 + half


@pytest.mark.parametrize("rows, cols", [(60, 200), (512, 300), (700, 700)])
@pytest.mark.parametrize("kind", ["decay", "lowrank"])
def test_spectra_that_fall(rows, cols, kind, ws):
    """Small singular values grow 3.4445-fold a step, and what is rounded in their directions with them."""
    g = gen(rows + cols)
    r = min(rows, cols)
    if kind == "decay":
        u = g.normal(size=(rows, r)) * np.logspace(0, -4, r) @ g.normal(size=(r, cols))
    else:
        u = g.normal(size=(rows, 4)) @ g.normal(size=(4, cols)) + 1e-3 * g.normal(size=(rows, cols))
    u = held(u, torch.float32)
    want, out = O.orthogonalise(u), torch.empty((rows, cols), device="cuda")
    B.gcn_orthogonalise(to_dev(u), out, ws)
    assert rel2(out.cpu().numpy(), want) <= 4 * rel2(f32_iteration(u), want) + 2.0 ** -21
    B.gcn_orthogonalise(to_dev(u), out, ws, prec=B.GCN_BF16)
    assert rel2(out.cpu().numpy(), want) <= 2.0 ** -8


@pytest.mark.parametrize("rows, cols", [(96, 700), (70, 2950), (2500, 96), (90, 20001), (30, 65536), (128, 4070), (4170, 128), (100, 333)])
def test_few_rows_and_many_columns(rows, cols, ws):
    """Tens to hundreds of workgroups a step, the last one's columns a part of its share."""
    u = np.random.default_rng(rows).normal(size=(rows, cols)).astype(np.float32)
    x = torch.from_numpy(u).cuda()
    got = B.gcn_orthogonalise(x, torch.empty_like(x), ws)
    again = B.gcn_orthogonalise(x, torch.empty_like(x), ws)
    assert torch.equal(got, again)
    want = O.orthogonalise(u)
    got = got.cpu().numpy().astype(np.float64)
    assert np.linalg.norm(got - want) <= O.error_bound(u) + 2.0 ** -24 * np.linalg.norm(want)
    assert rel2(got, want) <= 4 * rel2(f32_iteration(u), want) + 2.0 ** -21


@pytest.mark.parametrize("rows, cols", [(700, 700), (1024, 1100), (1500, 1500), (2300, 1030), (2050, 2300), (2500, 2500),
                                        (3000, 3300), (4096, 2816), (300, 9000), (4096, 4100)])
@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
def test_large_sides(rows, cols, prec, ws):
    """The other tile shapes, against the iteration in float64 on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    u = torch.randn((rows, cols), generator=g, device="cuda")
    out = torch.empty_like(u)
    B.gcn_orthogonalise(u, out, ws, prec=prec)
    x = u.double() / u.double().norm()
    x = x.T.contiguous() if rows > cols else x
    y = x.float()
    a, b, c = O.COEF
    for _ in range(5):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
        s = y @ y.T
        y = a * y + (b * s + c * (s @ s)) @ y
    x, y = (x.T, y.T) if rows > cols else (x, y)
    err, plain = ((v.double() - x).norm() / x.norm() for v in (out, y))
    assert float(err) <= (4 * float(plain) + 2.0 ** -21 if prec == B.GCN_F32 else 2.0 ** -8)


@pytest.mark.parametrize("steps", [1, 2, 7, 20])
def test_number_of_steps(steps, ws):
    u = held(gradient(gen(3), 90, 70), torch.float32)
    out, want = torch.empty((90, 70), device="cuda"), O.orthogonalise(u, steps)
    B.gcn_orthogonalise(to_dev(u), out, ws, steps=steps)
    assert rel2(out.cpu().numpy(), want) <= 4 * rel2(f32_iteration(u, steps), want) + 2.0 ** -21


def test_scale_does_not_matter(ws):
    """A power of two changes no bit, over the whole range of float32; the matrix may be its own result."""
    u = held(gradient(gen(4), 70, 90), torch.float32)
    u *= 2.0 ** -np.floor(np.log2(np.abs(u).max()))
    base, out = torch.empty((70, 90), device="cuda"), torch.empty((70, 90), device="cuda")
    B.gcn_orthogonalise(to_dev(u), base, ws)
    for k in (-100, -20, 60, 126):
        B.gcn_orthogonalise(to_dev(u * 2.0 ** k), out, ws)
        assert torch.equal(out, base), k
    same = to_dev(u)
    B.gcn_orthogonalise(same, same, ws)
    assert torch.equal(same, base)


@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
def test_zeros_and_values_that_are_not_finite(prec, ws):
    x = torch.zeros((40, 70), device="cuda")
    out = torch.full_like(x, 5.0)
    B.gcn_orthogonalise(x, out, ws, prec=prec)
    assert not out.any()
    x[3, 5] = 2.0 ** -149                              # one element alone: a matrix of rank one
    B.gcn_orthogonalise(x, out, ws, prec=prec)
    want = O.orthogonalise(np.array([[1.0]]))[0, 0]
    # x goes 1, 0.70, 1.11, 0.72, 1.09, 0.70.  Rounded by u = 2^-11 each, x, A and B put a step off by at most
    # (|b + 2 c x^2| x^3 (2 u + u) + 2 |b + c x^2| x^3 u < 5.5 u), and the slopes -1.14, 1.30, -1.26 and 0.76 there carry
    # it on: 5.5 u (1 + 0.76 + 0.96 + 1.25 + 1.43) < 30 u < 2^-6.  Pairs, which 40 rows take, have u = 2^-22
    assert abs(float(out[3, 5]) - want) < 2.0 ** -17
    assert int((out != 0).sum()) == 1
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.randn((40, 70), device="cuda")
        x[7, 9] = bad
        B.gcn_orthogonalise(x, out, ws, prec=prec)
        assert bool(torch.isnan(out).all())


# -------------------------------------------------------------------- update
def tensors(g, sides, gt, pad=0):
    out = []
    for r, c in sides:
        w, m = (held(g.normal(size=(r, c)), torch.float32) for _ in range(2))
        gr = held(gradient(g, r, c), gt)
        W, M, G = padded(r, c, torch.float32, pad), padded(r, c, torch.float32, 2 * pad), padded(r, c, gt, pad)
        W.copy_(to_dev(w))
        M.copy_(to_dev(m * 1e-2))
        G.copy_(to_dev(gr, gt))
        out.append((W, G, M, w, gr, M.to(torch.float64).cpu().numpy()))
    return out


def check_update(ts, lr, scales, prec, **kw):
    for (W, G, M, w, gr, m), s in zip(ts, scales):
        want_w, want_m = O.update(w, gr, m, lr, s, **kw)
        # one rounding of the momentum and one of its sum
        assert np.all(np.abs(M.cpu().numpy() - want_m) <= 2.0 ** -23 * (np.abs(m) + np.abs(gr)))
        u = gr + kw.get("momentum", 0.95) * want_m if kw.get("nesterov", True) else want_m
        o = np.linalg.norm(O.orthogonalise(u))
        tol = 4 * rel2(f32_iteration(u), O.orthogonalise(u)) + 2.0 ** -20 if prec == B.GCN_F32 else 2.0 ** -8
        assert np.linalg.norm(W.cpu().numpy() - want_w) <= lr * s * o * tol + 2.0 ** -22 * np.linalg.norm(w)


@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
@pytest.mark.parametrize("sides, pad", [([(50, 64)], 0), ([(602, 128), (602, 128), (256, 41), (1, 5)], 0),
                                        ([(33, 70), (70, 33), (64, 64), (300, 7)], 3)])
def test_update(sides, pad, gt, prec, ws):
    ts = tensors(gen(len(sides) + pad), sides, DT[gt], pad)
    scales = [0.5 + i for i in range(len(sides))]
    step = B.MuonStep([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts], scales=scales, weight_decay=0.1, prec=prec)
    step(0.02, ws)
    check_update(ts, 0.02, scales, prec, weight_decay=0.1)
    if pad:
        for W, *_ in ts:
            r, c = W.shape
            assert bool((W.as_strided((r, pad), (c + pad, 1), c) == 7.0).all())


@pytest.mark.parametrize("momentum, nesterov", [(0.0, True), (0.9, False), (0.9, True)])
def test_momentum_forms(momentum, nesterov, ws):
    ts = tensors(gen(8), [(40, 60), (60, 40)], torch.float32)
    step = B.MuonStep([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts], scales=[1.0, 2.0], momentum=momentum,
                      nesterov=nesterov)
    step(0.1, ws)
    check_update(ts, 0.1, [1.0, 2.0], B.GCN_F32, momentum=momentum, nesterov=nesterov)


def test_many_matrices_and_empty_ones(ws):
    """More than a launch takes, matrices without elements among them; every one as alone."""
    g = gen(11)
    sides = [(int(r), int(c)) for r, c in g.integers(1, 90, (37, 2))]
    sides[5], sides[20] = (0, 4), (4, 0)
    ts = tensors(g, sides, torch.float32)
    alone = [tuple(x.clone() for x in t[:3]) for t in ts]
    B.MuonStep([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts])(0.05, ws)
    for (W, G, M, *_), (w, gr, m) in zip(ts, alone):
        B.MuonStep([w], [gr], [m])(0.05, ws)
        if W.numel():
            assert float((W - w).norm()) <= 2.0 ** -20 * float(w.norm()) and torch.equal(M, m)


def test_column_ranges_of_one_array(ws):
    """W_self and W_neigh side by side, updated in one call."""
    g = gen(12)
    both, apart = to_dev(g.normal(size=(48, 80))), None
    G = [to_dev(gradient(g, 48, 40)) for _ in range(2)]
    M = [torch.zeros((48, 40), device="cuda") for _ in range(2)]
    apart = [both[:, :40].clone(), both[:, 40:].clone()]
    m2 = [m.clone() for m in M]
    B.MuonStep([both[:, :40], both[:, 40:]], G, M)(0.1, ws)
    B.MuonStep(apart, G, m2)(0.1, ws)
    assert torch.equal(both, torch.cat(apart, 1))


def test_a_second_update_moves_on(ws):
    ts = tensors(gen(13), [(64, 96)], torch.float32)
    W, G, M, w, gr, m = ts[0]
    step = B.MuonStep([W], [G], [M], scales=[1.0], momentum=0.5)
    for _ in range(3):
        step(0.1, ws)
        w, m = O.update(w, gr, m, 0.1, 1.0, momentum=0.5)
    assert rel2(W.cpu().numpy(), w) < 1e-5 and rel2(M.cpu().numpy(), m) < 1e-6


def test_captured_update(ws):
    """A captured step, replayed between eager work, moves as eager steps do."""
    ts = tensors(gen(14), [(130, 70), (40, 64)], torch.float32)
    ws.get(1 << 24)
    eager = [[x.clone() for x in t[:3]] for t in ts]
    step = B.MuonStep([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(0.05, ws)
    torch.cuda.synchronize()
    other = B.MuonStep([e[0] for e in eager], [e[1] for e in eager], [e[2] for e in eager])
    ws2 = B.Workspace()
    for _ in range(4):
        graph.replay()
        other(0.05, ws2)
        torch.cuda.synchronize()
        for (W, _, M, *_), (w, _, m) in zip(ts, eager):
            assert torch.equal(W, w) and torch.equal(M, m)


@pytest.mark.parametrize("rows, cols", [(602, 128), (64, 2000), (300, 400)])
def test_captured_in_each_way_of_working(rows, cols):
    """Two graphs with workspaces of their own, replayed in turn between eager calls of the same matrix."""
    x = to_dev(gradient(gen(31), rows, cols))
    ws, outs, graphs, spaces = B.Workspace(), [], [], []
    want = B.gcn_orthogonalise(x, torch.empty_like(x), ws)
    for _ in range(2):
        w, out = B.Workspace(), torch.empty_like(x)
        w.get(1 << 26)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                B.gcn_orthogonalise(x, out, w)
        outs.append(out)
        graphs.append(graph)
        spaces.append(w)
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.zero_()
            graph.replay()
            assert torch.equal(B.gcn_orthogonalise(x, torch.empty_like(x), ws), want)
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_another_stream(ws):
    """The calls follow the current stream: both ways of working, with their own workspaces at the same time."""
    a, b = to_dev(gradient(gen(20), 300, 200)), to_dev(gradient(gen(21), 60, 90))
    want = [B.gcn_orthogonalise(x, torch.empty_like(x), ws) for x in (a, b)]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(x) for x in (a, b)]
    spaces = [B.Workspace() for _ in range(2)]
    for w in spaces:
        w.get(1 << 24)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, w, x, o in zip(streams, spaces, (a, b), got):
            with torch.cuda.stream(s):
                B.gcn_orthogonalise(x, o, w)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
