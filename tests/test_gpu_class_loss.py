"""The many-class loss on the GPU against its float64 definition."""
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


def inputs(n, f, C, dtype, seed=0, bias=True, unlabelled=0.1, scale=2.0):
    g = np.random.default_rng(seed + n + 3 * f + 7 * C)
    t = DT[dtype]
    hold = lambda x: torch.from_numpy(np.asarray(x, np.float32)).to(t)
    H, W = hold(np.maximum(g.normal(size=(n, f)), 0)), hold(g.normal(size=(f, C)) * scale / np.sqrt(f))
    b = torch.from_numpy(g.normal(size=C).astype(np.float32)) if bias else None
    lab = g.integers(0, C, n).astype(np.int32)
    lab[g.random(n) < unlabelled] = -1
    return H, W, b, lab


class Out:
    def __init__(self, n, f, C, t, grad=True, pad=0):
        e = lambda *s, dt=torch.float32: torch.full(s, 7.0, dtype=dt, device="cuda")
        self.loss, self.rows = e(1), e(n)
        self.dH = e(n, f + pad, dt=t)[:, :f] if grad else None
        self.dW, self.db = (e(f, C, dt=t), e(C)) if grad else (None, None)

    def all(self):
        return [x for x in (self.loss, self.rows, self.dH, self.dW, self.db) if x is not None]


def call(H, W, b, lab, out, ws=None, stream=None):
    B.gcn_class_loss(H, W, b, lab, out.loss, ws or B.Workspace(), row_loss=out.rows, dHL=out.dH, dW_pred=out.dW,
                     db_pred=out.db, stream=stream)


def np64(t):
    return t.to(torch.float64).cpu().numpy()


def check(H, W, b, lab, out, dtype):
    """Against the definition, element by element.  A logit's sum of f products
    is off by (f + 4) 2^-23 of their magnitudes at most (bfloat16: the products
    are exact); exp and log add 2^-20 of the distance from the maximum, which
    is below 64 here.  G moves by twice that; bfloat16 G is rounded by 2^-8
    before the two products, and the results by 2^-8."""
    h, w = np64(H), np64(W)
    bb = None if b is None else np64(b)
    loss, rows, dH, dW, db, G = R.class_loss(np.where(np.isfinite(h), h, 0.0), w, bb, lab)
    n, f = h.shape
    has = (lab >= 0) & (lab < w.shape[1])
    hz = np.where(has[:, None], h, 0.0)
    mag = np.abs(hz) @ np.abs(w) + (0.0 if bb is None else np.where(np.isfinite(bb), np.abs(bb), 0.0))
    dx = (f + 4) * 2.0 ** -23 * mag.max(1, initial=0.0) + 64 * 2.0 ** -20
    assert np.all(np.abs(np64(out.rows) - rows) <= 2 * dx + 2.0 ** -22 * np.abs(rows))
    assert np.all(np64(out.rows)[~has] == 0.0)
    assert abs(float(out.loss) - loss) <= 2 * dx.max(initial=0.0) + 2.0 ** -22 * abs(loss)
    if out.dH is None:
        return
    count = max(1, int(has.sum()))
    # the error of p (1 - onehot adds a rounding of p against 1, 2^-24)
    dG = np.where(has[:, None], (np.abs(G) + 2.0 ** -23 / count) * (4 * dx[:, None] + 2.0 ** -22), 0.0)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    g1 = dG + half * (np.abs(G) + dG)
    C = w.shape[1]
    tH = g1 @ np.abs(w).T + (C + 70) * 2.0 ** -23 * (np.abs(G) @ np.abs(w).T)
    tW = np.abs(hz).T @ g1 + (n + 70) * 2.0 ** -23 * (np.abs(hz).T @ np.abs(G))
    tb = dG.sum(0) + (n + 70) * 2.0 ** -23 * np.abs(G).sum(0)
    tH, tW = tH + half * (np.abs(dH) + tH), tW + half * (np.abs(dW) + tW)
    for got, want, tol, name in ((out.dH, dH, tH, "dH"), (out.dW, dW, tW, "dW"), (out.db, db, tb, "db")):
        err = np.abs(np64(got) - want)
        assert np.all(err <= tol + 1e-37), (name, float(np.max(err / (tol + 1e-37))))
    assert np.all(np64(out.dH)[~has] == 0.0)


SIZES = [(1, 1, 1), (1, 64, 3), (2, 3, 2), (17, 50, 41), (64, 64, 128), (65, 130, 129), (130, 96, 1000), (300, 257, 517),
         (33, 512, 4099), (2100, 200, 5300), (2600, 1030, 4500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, f, C", SIZES)
def test_loss_and_gradient(n, f, C, dtype):
    H, W, b, lab = inputs(n, f, C, dtype)
    if n > 4:
        lab[1], lab[2] = C, -2 ** 31          # no class either
        lab[3] = C - 1
    pad = 3 if n == 65 else 0
    out = Out(n, f, C, DT[dtype], pad=pad)
    Hd = torch.full((n, f + pad), 3.0, dtype=DT[dtype], device="cuda")[:, :f]
    Hd.copy_(H)
    call(Hd, W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    check(H, W, b, lab, out, dtype)
    if pad:
        assert float(torch.as_strided(out.dH, (n, f + pad), (f + pad, 1))[:, f:].min()) == 7.0
    ev = Out(n, f, C, DT[dtype], grad=False)   # evaluation: the same losses
    call(Hd, W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), ev)
    assert torch.equal(ev.loss, out.loss) and torch.equal(ev.rows, out.rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_bias_and_same_label_everywhere(dtype):
    H, W, _, lab = inputs(90, 70, 333, dtype, bias=False, unlabelled=0.0)
    lab[:] = 332
    out = Out(90, 70, 333, DT[dtype])
    call(H.cuda(), W.cuda(), None, torch.from_numpy(lab).cuda(), out)
    check(H, W, None, lab, out, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_label_reach_nothing(dtype):
    """NaN and infinities in HL where there is no label; and no label at all."""
    n, f, C = 70, 40, 300
    H, W, b, lab = inputs(n, f, C, dtype, unlabelled=0.4)
    H[torch.from_numpy(lab < 0)] = float("nan")
    H[int(np.nonzero(lab < 0)[0][0]), 3] = float("inf")
    out = Out(n, f, C, DT[dtype])
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    check(H, W, b, lab, out, dtype)
    lab[:] = -1
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    assert all(float(x.abs().max()) == 0.0 for x in out.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("-inf"), float("inf"), float("nan")])
def test_rows_without_a_label_and_no_logit_left(dtype, value):
    """Without a label every result is 0 whatever the logits are: all minus infinity, plus infinity, NaN."""
    n, f, C = 150, 40, 270
    H, W, b, lab = inputs(n, f, C, dtype)
    b[:] = value
    lab[:] = -1
    out = Out(n, f, C, DT[dtype])
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    assert all(float(x.abs().max()) == 0.0 for x in out.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_classes_switched_off(dtype):
    """A bias of minus infinity or of the type's lowest value; whole column tiles of them, the first and the last."""
    n, f, C = 40, 32, 700
    H, W, b, lab = inputs(n, f, C, dtype, unlabelled=0.0)
    b[:300] = float("-inf")
    b[500:] = torch.finfo(torch.float32).min
    lab[:] = np.random.default_rng(1).integers(300, 500, n)
    out = Out(n, f, C, DT[dtype])
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    keep = slice(300, 500)
    small = Out(n, f, 200, DT[dtype])
    small.loss, small.rows, small.dH = out.loss, out.rows, out.dH
    small.dW, small.db = out.dW[:, keep], out.db[keep]
    check(H, W[:, keep], b[keep], lab - 300, small, dtype)
    off = torch.cat([out.dW[:, :300], out.dW[:, 500:]], 1)
    assert float(off.abs().max()) == 0.0 and float(out.db[:300].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_that_are_not_finite_are_seen(dtype):
    n, f, C = 9, 16, 50
    H, W, b, lab = inputs(n, f, C, dtype, unlabelled=0.0)
    H[4, 2] = float("nan")
    out = Out(n, f, C, DT[dtype])
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    r = np64(out.rows)
    assert np.isnan(r[4]) and np.isfinite(np.delete(r, 4)).all() and np.isnan(float(out.loss))
    assert torch.isnan(out.dH[4]).all() and torch.isfinite(out.dH[:4]).all()


def test_far_logits():
    """Logits hundreds apart: one probability of 1, the others underflow, the loss stays exact."""
    n, f, C = 8, 8, 260
    H = torch.eye(8, dtype=torch.float32) * 1000
    W = torch.zeros((f, C))
    W[:, 0], W[:, 259] = 1.0, -1.0
    lab = np.array([0, 259, 1, 0, 259, 1, 0, 0], np.int32)
    for dtype in ("f32", "bf16"):
        out = Out(n, f, C, DT[dtype])
        call(H.to(DT[dtype]).cuda(), W.to(DT[dtype]).cuda(), None, torch.from_numpy(lab).cuda(), out)
        assert np.array_equal(np64(out.rows), np.array([0, 2000, 1000, 0, 2000, 1000, 0, 0.0]))


@pytest.mark.parametrize("dtype, n, f, C", [("bf16", 300000, 16, 1500), ("f32", 60000, 8, 2500),
                                            ("f32", 140000, 32, 1100), ("bf16", 600000, 64, 712)])
def test_several_pieces(dtype, n, f, C):
    """Sizes that are cut into pieces of the classes, the last one ragged, against torch in float64 on the GPU."""
    t = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    H = torch.relu(torch.randn(n, f, generator=g, device="cuda")).to(t)
    W = torch.randn(f, C, generator=g, device="cuda").to(t)
    lab = torch.randint(-1, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    b = torch.randn(C, generator=g, device="cuda")
    out = Out(n, f, C, t)
    call(H, W, b, lab, out)
    has = lab >= 0
    dW, db, total, count = torch.zeros(f, C, dtype=torch.float64, device="cuda"), 0.0, 0.0, int(has.sum())
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for r in torch.split(torch.arange(n, device="cuda"), 20000):
        h, y = H[r].double(), has[r]
        logp = torch.log_softmax(h @ W.double() + b.double(), 1)
        at = lab[r].long().clamp(min=0)
        rows = torch.where(y, -logp.gather(1, at[:, None])[:, 0], 0.0)
        # logits below 2^6 in magnitude: (f + 4) 2^-23 2^6 and exp's 2^-14
        assert float((out.rows[r].double() - rows).abs().max()) < 1e-3
        G = logp.exp()
        G[torch.arange(len(r), device="cuda"), at] -= 1
        G = G * y[:, None] / count
        dH = G @ W.double().T
        tol = (1e-3 + half) * (G.abs() @ W.double().abs().T) + half * dH.abs()
        assert bool(((out.dH[r].double() - dH).abs() <= tol).all())
        dW += (h * y[:, None]).T @ G
        db = db + G.sum(0)
        total += float(rows.sum())
    assert abs(float(out.loss) - total / count) < 1e-4
    mean = dW.abs().mean()
    assert float((out.dW.double() - dW).abs().max()) < (2e-3 + 2 * half) * float(mean + dW.abs().max())
    assert float((out.db.double() - db).abs().max()) < 1e-3 * float(db.abs().max())


def test_gradient_against_differences():
    """The loss's change along directions of H, W and b, float32: h^2 of the third derivative and the loss's own
    2^-22 / h."""
    n, f, C = 40, 24, 90
    H, W, b, lab = inputs(n, f, C, "f32", unlabelled=0.2)
    labd = torch.from_numpy(lab).cuda()
    out = Out(n, f, C, torch.float32)
    call(H.cuda(), W.cuda(), b.cuda(), labd, out)
    g = torch.Generator().manual_seed(2)
    D = [torch.randn(x.shape, generator=g) for x in (H, W, b)]
    want = sum(float((np64(a) * np64(d)).sum()) for a, d in zip((out.dH, out.dW, out.db), D))
    h = 2.0 ** -7
    val = []
    for s in (h, -h):
        o = Out(n, f, C, torch.float32, grad=False)
        call((H + s * D[0]).cuda(), (W + s * D[1]).cuda(), (b + s * D[2]).cuda(), labd, o)
        val.append(float(o.loss))
    # a logit moves by t (|h| |D1| + |D0| |w| + |D2|) + t^2 |D0| |D1| along D, below 2^5 each per unit of t
    assert abs((val[0] - val[1]) / (2 * h) - want) < h * h * 2.0 ** 12 / n + 2.0 ** -21 * 8 / h


def test_no_rows():
    for dtype in ("f32", "bf16"):
        out = Out(0, 12, 30, DT[dtype])
        call(torch.empty((0, 12), dtype=DT[dtype], device="cuda"), torch.ones((12, 30), dtype=DT[dtype], device="cuda"),
             None, torch.empty(0, dtype=torch.int32, device="cuda"), out)
        assert float(out.loss) == 0.0 and float(out.dW.abs().max()) == 0.0 and float(out.db.abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_streams_and_graphs(dtype):
    n, f, C = 500, 96, 2100
    sets = [inputs(n, f, C, dtype, seed=s) for s in range(3)]
    H, W, b, lab = [x.cuda() if torch.is_tensor(x) else torch.from_numpy(x).cuda() for x in sets[0]]
    out, ws = Out(n, f, C, DT[dtype]), B.Workspace()
    ws.get(256 << 20)
    call(H, W, b, lab, out, ws)
    torch.cuda.synchronize()
    side, again = torch.cuda.Stream(), Out(n, f, C, DT[dtype])
    ws2 = B.Workspace()
    ws2.get(256 << 20)
    torch.cuda.synchronize()
    call(H, W, b, lab, again, ws2, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out.all(), again.all()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(H, W, b, lab, out, ws)
    for k in (1, 2, 0, 1):
        for dst, src in zip((H, W, b, lab), sets[k]):
            dst.copy_(src if torch.is_tensor(src) else torch.from_numpy(src))
        graph.replay()
        eager = Out(n, f, C, DT[dtype])
        call(H, W, b, lab, eager, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out.all(), eager.all()))
