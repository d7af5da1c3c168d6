"""Whole updates through every way of working, the largest tiles included:
momentum, weight decay and the stores into W, also transposed and past whole
vectors, against float64 on the GPU; calls that mix sizes."""
import numpy as np
import pytest
import torch

from oracle import muon as O
from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, MU, DECAY = 0.05, 0.95, 0.5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture()
def ws():
    return B.Workspace()


def iterate(u, dtype, steps=5):
    """The iteration in `dtype` products."""
    x = u / u.norm()
    x = x.T.contiguous() if x.shape[0] > x.shape[1] else x
    x = x.to(dtype)
    a, b, c = O.COEF
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def view(rows, cols, dtype, pad):
    return torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")[:, :cols]


def matrices(sides, gt, pad, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for r, c in sides:
        W, M, G = view(r, c, torch.float32, pad), view(r, c, torch.float32, pad and pad + 2), view(r, c, gt, pad)
        for t in (W, M, G):
            t.copy_(torch.randn((r, c), generator=g, device="cuda"))
        out.append((W, G, M))
    return out


def untouched(t, pad):
    r, c = t.shape
    return not pad or bool((t.as_strided((r, pad), (c + pad, 1), c) == 7.0).all())


def check(sides, gt, prec, pad, ws):
    ts = matrices(sides, DT[gt], pad, sum(r + 3 * c for r, c in sides))
    before = [(W.clone(), M.clone()) for W, _, M in ts]
    # (updates of the weights' own size: a factor of sqrt(max) makes an orthogonal matrix's elements about one)
    scales = [max(s) ** 0.5 / LR for s in sides]
    step = B.MuonStep([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts], scales=scales, momentum=MU,
                      weight_decay=DECAY, prec=prec)
    step(LR, ws)
    for (W, G, M), (w, m), s in zip(ts, before, scales):
        want_m = MU * m.double() + G.double()
        # one rounding of the momentum, one of its factor and one of their sum
        assert bool(((M.double() - want_m).abs() <= 2.0 ** -23 * (m.abs().double() + G.abs().double())).all())
        u = G.double() + MU * want_m
        o, p = iterate(u, torch.float64), iterate(u, torch.float32).double()
        want = (1 - LR * DECAY) * w.double() - LR * s * o
        tol = 4 * float((p - o).norm()) + 2.0 ** -20 * float(o.norm()) if prec == B.GCN_F32 else 2.0 ** -8 * float(o.norm())
        assert float((W.double() - want).norm()) <= LR * s * tol + 2.0 ** -22 * float(w.double().norm())
        assert untouched(W, pad) and untouched(M, pad and pad + 2) and untouched(G, pad)
    if len(sides) == 1:
        # element by element: alone, a matrix's update is the orthogonalised matrix of the same kernels, bit for bit
        # (U's one rounding, of an exact product's sum, is the same from 64 bits)
        W, G, M = ts[0]
        u = (G.double() + float(np.float32(MU)) * M.double()).float()
        o = B.gcn_orthogonalise(u, torch.empty_like(u), ws, prec=prec)
        w, f = before[0][0], LR * scales[0]
        want = (1 - LR * DECAY) * w.double() - f * o.double()
        # roundings of both factors, of a product and of the sum
        assert bool(((W.double() - want).abs() <= 2.0 ** -22 * (w.abs().double() + f * o.abs().double())).all())
    # and again from the same start: the same bits
    got = [W.clone() for W, _, _ in ts]
    for (W, _, M), (w, m) in zip(ts, before):
        W.copy_(w)
        M.copy_(m)
    step(LR, ws)
    assert all(torch.equal(W, x) for (W, _, _), x in zip(ts, got))


SIDES = [(50, 64), (64, 2000), (2000, 33), (602, 128), (128, 4070), (700, 500), (500, 701), (1030, 2300), (2300, 1030),
         (2000, 2503), (3000, 3300), (3301, 3000), (4096, 4096)]


@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
@pytest.mark.parametrize("gt, pad", [("f32", 0), ("bf16", 3)])
@pytest.mark.parametrize("rows, cols", SIDES)
def test_update_of_every_tile(rows, cols, gt, pad, prec, ws):
    check([(rows, cols)], gt, prec, pad, ws)


@pytest.mark.parametrize("prec", [B.GCN_F32, B.GCN_BF16])
@pytest.mark.parametrize("sides", [[(4096, 4096), (602, 128), (50, 64)], [(50, 64), (64, 2000), (33, 5)],
                                   [(1, 1), (3000, 3300), (2000, 33)], [(512, 512), (300, 128), (128, 300), (7, 900)]])
def test_unlike_sizes_in_one_call(sides, prec, ws):
    """The widest decides for all of its launch: each is right all the same, and the call repeats its bits."""
    check(sides, "f32", prec, 0, ws)
    check(sides[::-1], "bf16", prec, 1, ws)
