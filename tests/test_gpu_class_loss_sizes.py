"""The many-class loss at the sizes of its large tiles: several pieces read in
place, weight gradients stored straight from one part, few rows of very many
classes; element by element against float64."""
import pytest
import torch

from tests.gpu_util import require_gpu
from tests.test_gpu_class_loss import DT, Out, call, check, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


# (31,990 x 1280: pieces of 8192 and 8128 classes, read in place, all four products on large tiles, dW in one part;
# 16,000 x 300, 17,001 classes: copied pieces; 60,000 rows float32: two pieces; 3000 x 640: one piece, in place)
@pytest.mark.parametrize("dtype, n, f, C", [("bf16", 31990, 1280, 16320), ("bf16", 16000, 300, 17001),
                                            ("f32", 60000, 40, 2500), ("bf16", 3000, 640, 12800),
                                            ("f32", 3000, 640, 6400)])
def test_large_tiles_and_pieces(dtype, n, f, C):
    t = DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(n + f)
    H = torch.relu(torch.randn(n, f, generator=g, device="cuda")).to(t)
    W = (torch.randn(f, C, generator=g, device="cuda") * (2.0 / f ** 0.5)).to(t)
    b = torch.randn(C, generator=g, device="cuda")
    lab = torch.randint(-C // 8, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    out, ev = Out(n, f, C, t), Out(n, f, C, t, grad=False)
    call(H, W, b, lab, out)
    call(H, W, b, lab, ev)
    assert torch.equal(ev.loss, out.loss) and torch.equal(ev.rows, out.rows)
    has = lab >= 0
    count = int(has.sum())
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    Wd, Wt = W.double(), W.double().T.contiguous()
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")
    dW, tW, mW, db, tb, total, far = zero(f, C), zero(f, C), zero(f, C), zero(C), zero(C), 0.0, 0.0
    for r in torch.split(torch.arange(n, device="cuda"), 4096):
        h, y = H[r].double() * has[r, None], has[r]
        logp = torch.log_softmax(h @ Wd + b.double(), 1)
        at = lab[r].long().clamp(min=0)
        rows = torch.where(y, -logp.gather(1, at[:, None])[:, 0], 0.0)
        # the errors of check(): a logit's f + 4 roundings, exp and log 2^-20 of at most 64
        dx = (f + 4) * 2.0 ** -23 * (h @ Wd.abs() + b.double().abs()).amax(1) + 64 * 2.0 ** -20
        assert bool(((out.rows[r].double() - rows).abs() <= 2 * dx + 2.0 ** -22 * rows).all())
        G = logp.exp()
        G[torch.arange(len(r), device="cuda"), at] -= 1
        G *= y[:, None] / count
        dG = torch.where(y[:, None], (G.abs() + 2.0 ** -23 / count) * (4 * dx[:, None] + 2.0 ** -22), 0.0)
        tb += dG.sum(0) + (n + 70) * 2.0 ** -23 * G.abs().sum(0)
        dG = dG + half * (G.abs() + dG)
        dH = G @ Wt
        tol = dG @ Wt.abs() + (C + 70) * 2.0 ** -23 * (G.abs() @ Wt.abs())
        tol = tol + half * (dH.abs() + tol)
        err = (out.dH[r].double() - dH).abs()
        assert bool((err <= tol + 1e-37).all())
        # rounded twice by half a step (bfloat16; root mean square below 2^-8 / sqrt(3) each), or by float32's sums
        assert float(err.norm()) <= (half + 2.0 ** -16) * float(dH.norm())
        ht = h.T.contiguous()
        dW += ht @ G
        tW += ht.abs() @ dG
        mW += ht.abs() @ G.abs()
        db += G.sum(0)
        total += float(rows.sum())
        far = max(far, float(dx.max()))
    assert abs(float(out.loss) - total / count) <= 2 * far + 2.0 ** -22 * total / count
    tol = tW + (n + 70) * 2.0 ** -23 * mW
    tol = tol + half * (dW.abs() + tol)
    err = (out.dW.double() - dW).abs()
    assert bool((err <= tol + 1e-37).all())
    assert float(err.norm()) <= (half + 2.0 ** -16) * float(dW.norm())
    assert bool(((out.db.double() - db).abs() <= tb + 1e-37).all())
    assert float((out.db.double() - db).norm()) <= 2.0 ** -16 * float(db.norm())
    assert float(out.dH[~has].abs().max()) == 0.0 and float(out.rows[~has].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, f, C", [(17, 256, 45056), (1, 200, 50001), (64, 64, 41000), (3, 520, 41215)])
def test_few_rows_of_very_many_classes(n, f, C, dtype):
    """Tiles that a few rows fill in part only."""
    H, W, b, lab = inputs(n, f, C, dtype)
    lab[0] = C - 1
    out = Out(n, f, C, DT[dtype])
    call(H.cuda(), W.cuda(), b.cuda(), torch.from_numpy(lab).cuda(), out)
    check(H, W, b, lab, out, dtype)
