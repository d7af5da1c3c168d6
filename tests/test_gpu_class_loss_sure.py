"""The many-class loss of rows that are sure of their label: small losses at
large logits, against float64."""
import numpy as np
import pytest
import torch

from oracle import rows8 as R
from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GAPS = [0.0, 0.5, 1.0, 5.0, 10.0, 11.0, 14.0]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def np64(t):
    return t.to(torch.float64).cpu().numpy()


def operands(gaps, C, other):
    """Row i: logits 1000 for class 0, 1000 - gaps[i] for class `other`, -1000 for the rest; every factor and every
    product is exact in either type."""
    H = np.stack([np.full(len(gaps), 8.0), np.asarray(gaps)], 1)
    W = np.zeros((2, C))
    W[0] = -125.0
    W[:, 0], W[:, other] = (125.0, 0.0), (125.0, -1.0)
    return H, W


def run(H, W, lab, dtype):
    t, (n, f), C = DT[dtype], H.shape, W.shape[1]
    e = lambda *s, dt=torch.float32: torch.full(s, 7.0, dtype=dt, device="cuda")
    loss, rows, dH, dW, db = e(1), e(n), e(n, f, dt=t), e(f, C, dt=t), e(C)
    dev = lambda x: torch.from_numpy(x).to("cuda").to(t)
    B.gcn_class_loss(dev(H), dev(W), None, torch.from_numpy(lab).cuda(), loss, B.Workspace(), row_loss=rows, dHL=dH,
                     dW_pred=dW, db_pred=db)
    return [np64(x) for x in (loss, rows, dH, dW, db)]


def check(H, W, lab, dtype):
    """e^-g is off by 2^-18 of itself (the exponent 1.44 g, below 21, is rounded twice by 2^-24, and the sum's join
    does it once more), the sum in [1, 2] by 2^-24 a step, its logarithm and the difference of two logits by 2^-23 of
    themselves: nowhere does the logits' size of 1000 enter.  p and 1 - p move as much; G is rounded to bfloat16 by
    2^-8 ahead of the two products in that type, and their results are."""
    loss, rows, dH, dW, db = run(H, W, lab, dtype)
    loss_, rows_, dH_, dW_, db_, G = R.class_loss(H, W, None, lab)
    n = len(lab)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = 2.0 ** -22 + 2.0 ** -18 * np.exp(-np.abs(H[:, 1])) + 2.0 ** -22 * rows_
    assert np.all(np.abs(rows - rows_) <= tol), float(np.max(np.abs(rows - rows_) / tol))
    assert abs(loss[0] - loss_) <= tol.mean() + 2.0 ** -23 * loss_
    dG = np.where(G != 0, 2.0 ** -21 / n + 2.0 ** -18 * np.abs(G), 0.0)
    sums = (n + 70) * 2.0 ** -23
    tb = dG.sum(0) + sums * np.abs(G).sum(0)
    assert np.all(np.abs(db - db_) <= tb), float(np.max(np.abs(db - db_) - tb))
    dG = dG + half * (np.abs(G) + dG)
    tW, tH = np.abs(H).T @ dG + sums * (np.abs(H).T @ np.abs(G)), dG @ np.abs(W).T + sums * (np.abs(G) @ np.abs(W).T)
    for got, want, t in ((dW, dW_, tW), (dH, dH_, tH)):
        t = t + half * (np.abs(want) + t)
        assert np.all(np.abs(got - want) <= t), float(np.max(np.abs(got - want) - t))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("label", [0, 1])
@pytest.mark.parametrize("C, other", [(2, 1), (700, 650)])
def test_one_sure_row(dtype, label, C, other):
    for g in GAPS:
        H, W = operands([g], C, other)
        check(H, W, np.array([other if label else 0], np.int32), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, C, other", [(70, 300, 299), (1100, 700, 650), (1500, 9000, 8100)])
def test_many_sure_rows(dtype, n, C, other):
    """Sizes whose statistics are joined by the loss's workgroup, by their own kernel, and of large tiles."""
    H, W = operands(np.resize(GAPS, n), C, other)
    lab = np.where(np.arange(n) % 3 == 0, other, 0).astype(np.int32)
    lab[np.arange(n) % 11 == 5] = -1
    check(H, W, lab, dtype)
