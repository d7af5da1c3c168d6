"""The training loop with the orthogonalised update: each iteration's update
against float64 on the GPU's own gradients, and the layout it works on."""
import numpy as np
import pytest
import torch

from oracle import muon as OM
from oracle import optim as OO
from tests.gpu_util import rel_inf, require_gpu
from paper_1810_11899_amd import binding as B
from paper_1810_11899_amd import synth
from paper_1810_11899_amd.train import FlatModel, SamplerConfig, Trainer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("f, dims", [(24, [(24, 16), (32, 16)]), (23, [(23, 64), (128, 40)])])
def test_each_iterations_update(f, dims):
    tg = synth.training_graph(3000, 16, f, 7, seed=3)
    tr = Trainer(tg, dims, SamplerConfig(m=40, n=300, eta=2.0, cap=20, pool=3, seed=5), lr=0.01, optimizer="muon")
    mdl = tr.model
    for it in range(1, 6):                        # crosses a pool refill
        P, M, V = mdl.host_tensors(), mdl.host_tensors(mdl.m), mdl.host_tensors(mdl.v)
        tr.step()
        torch.cuda.synchronize()
        G, P2, M2 = mdl.host_tensors(mdl.grads), mdl.host_tensors(), mdl.host_tensors(mdl.m)
        for k in P:
            if k.startswith("W_") and k != "W_pred":
                s = 0.2 * np.sqrt(max(P[k].shape))
                w, m = OM.update(P[k], G[k], M[k], 0.01, s)
                # the update within the iteration's own bound, W within its rounding
                u = G[k].astype(np.float64) + 0.95 * m
                assert np.linalg.norm(P2[k] - w) <= 0.01 * s * OM.error_bound(u) + 2.0 ** -22 * np.linalg.norm(w), (it, k)
            else:
                w, m, _ = OO.adam(P[k], G[k], M[k], V[k], it, 0.01)
                assert rel_inf(P2[k], w) <= 1e-6, (it, k)
            assert rel_inf(M2[k], m) <= 1e-6, (it, k)
        assert all(not p.any() for p in mdl.padding_rows())
    assert np.isfinite(tr.loss_history()).all()


def test_layouts_hold_the_same_model():
    a = FlatModel([(23, 16), (32, 8)], 5, "cuda", seed=2)
    b = FlatModel([(23, 16), (32, 8)], 5, "cuda", seed=2, matrices_first=True)
    for (k, x), y in zip(a.host_tensors().items(), b.host_tensors().values()):
        assert np.array_equal(x, y), k
    assert a.total == b.total
    ends = [o + int(np.prod(s)) for o, s in zip(b.offsets, b.shapes)]
    assert all(ends[i] <= b.tail for i in b.matrices)
    assert all(b.offsets[i] >= b.tail for i in range(len(b.shapes)) if i not in b.matrices)
    assert [tuple(v.shape) for v in b.matrix_views(b.params)] == [(23, 16), (23, 16), (32, 8), (32, 8)]


def test_other_optimizers_are_refused():
    with pytest.raises(ValueError, match="optimizer"):
        Trainer(None, [], SamplerConfig(), optimizer="sgd")


def test_a_layer_trained_in_4_bits():
    """A run of the operators together: every step packs the weights in both orientations, multiplies forward, takes
    the ReLU derivative and the bias gradient while packing dZ both ways, forms dX and dW, and updates W."""
    n, K, N = 300, 130, 70
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    x = torch.relu(torch.randn((n, K), generator=g, device="cuda"))
    W = torch.randn((K, N), generator=g, device="cuda") * K ** -0.5
    b = torch.zeros(N, device="cuda")
    M, dW, dX = torch.zeros_like(W), torch.empty_like(W), torch.empty_like(x)
    goal = torch.randn((n, N), generator=g, device="cuda")
    Y, db, ws = torch.empty((n, N), device="cuda"), torch.empty(N, device="cuda"), B.Workspace()
    X4, X4T, W4, W4T = B.Rows4(n, K), B.Rows4(K, n), B.Rows4(K, N), B.Rows4(N, K)
    dZ4, dZ4T = B.Rows4(n, N), B.Rows4(N, n)
    B.gcn_rows4_pack(x, ws, out=X4, out_t=X4T)
    step = B.MuonStep([W], [dW], [M], scales=[1.0], weight_decay=0.01)

    def values(r):
        v = torch.empty((r.n, r.f), device="cuda")
        return B.gcn_rows4_unpack(r, v).double()

    for it in range(4):
        B.gcn_rows4_pack(W, ws, out=W4, out_t=W4T)
        B.gcn_rows4_product(X4, W4T, Y, ws, bias=b, relu=True)
        dY = (Y - goal) / n
        B.gcn_rows4_pack(dY, ws, out=dZ4, out_t=dZ4T, mask=Y, colsum=db)
        B.gcn_rows4_product(dZ4, W4, dX, ws)
        B.gcn_rows4_product(X4T, dZ4T, dW, ws)
        dz = torch.where(Y > 0, dY, torch.zeros_like(dY)).double()
        # sums of K, N and n exact products, each addition within 2^-22 of the magnitudes so far
        for got, p, q in ((Y, X4, W4T), (dX, dZ4, W4), (dW, X4T, dZ4T)):
            p, q = values(p), values(q)
            want = p @ q.T
            if got is Y:
                want = torch.relu(want + b.double())
            assert bool(((got.double() - want).abs() <= 70 * 2.0 ** -22 * (p.abs() @ q.abs().T + b.double().abs().max())).all())
        assert bool(((db.double() - dz.sum(0)).abs() <= n * 2.0 ** -24 * dz.abs().sum(0)).all())
        # a packed value is off by at most a quarter of its block's largest (half the step of 2 in 4 .. 6, over 3 at least)
        assert float((values(dZ4) - dz).norm()) < 0.25 * float(dz.norm())
        w0, m0 = W.cpu().numpy(), M.cpu().numpy()
        step(0.05, ws)
        w, m = OM.update(w0, dW.cpu().numpy(), m0, 0.05, 1.0, weight_decay=0.01)
        u = dW.cpu().numpy().astype(np.float64) + 0.95 * m
        assert np.linalg.norm(W.cpu().numpy() - w) <= 0.05 * OM.error_bound(u) + 2.0 ** -22 * np.linalg.norm(w)
        b -= 0.05 * db
