"""The 8-bit step as a training loop runs it: weights that change between the
steps, the memory it takes, and its input gradients against unrounded ones."""
import numpy as np
import pytest
import torch

from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B
from paper_1810_11899_amd import synth
from paper_1810_11899_amd.runner import StepRunner, StepRunner8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def outputs(r):
    return ([r.loss, r.row_loss, r.dHL, r.dW_pred, r.db_pred] + r.dWs + r.dWn + r.db + [d for d in r.dH if d is not None])


def workload(seed=2):
    # (a layer of 40 columns: the halves of [W_self || W_neigh] share blocks)
    return synth.custom(400, "rmat", 7, [(30, 40), (80, 64), (128, 24)], head="ce", classes=90, seed=seed)


def test_updated_weights_reach_both_directions():
    wl = workload()
    r = StepRunner8(wl)
    r.step()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    for l, (Ws, Wn, b) in zip(wl.layers, r.W):
        for t, name in ((Ws, "W_self"), (Wn, "W_neigh"), (b, "bias")):
            t.add_(torch.randn(t.shape, generator=gen, device="cuda"), alpha=0.5)
            setattr(l, name, t.cpu().numpy())
    r.step()
    fresh = StepRunner8(wl)
    fresh.step()
    torch.cuda.synchronize()
    for a, b in zip(outputs(r), outputs(fresh)):
        assert torch.equal(a, b)


def test_adam_on_the_steps_own_weights():
    """The layers' tensors go into the optimizer as they are, on a stream of the caller's: two training steps give what
    runners built from the updated weights give."""
    wl = workload()
    r = StepRunner8(wl)
    r.ws.get(64 << 20)
    moments = [[(torch.zeros_like(p), torch.zeros_like(p)) for p in w] for w in r.W]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for k in (1, 2):
        r.step(stream)
        stream.synchronize()
        fresh = StepRunner8(wl)
        fresh.step()
        torch.cuda.synchronize()
        for a, b in zip(outputs(r), outputs(fresh)):
            assert torch.equal(a, b)
        for w, g, mv in zip(r.W, zip(r.dWs, r.dWn, r.db), moments):
            for p, d, (m, v) in zip(w, g, mv):
                B.gcn_adam_update(p, d, m, v, 0.05, k, stream=stream)
        stream.synchronize()
        for l, w in zip(wl.layers, r.W):
            l.W_self, l.W_neigh, l.bias = [p.cpu().numpy() for p in w]


@pytest.mark.parametrize("layers", [[(30, 40)], [(30, 40), (80, 64)], [(30, 40), (80, 150), (300, 24), (48, 33)]])
def test_shared_buffers_give_the_same_step(layers):
    """keep_gradients or not: the same bits, and dH of the lowest layer that has one."""
    wl = synth.custom(500, "er", 9, layers, head="ce", classes=70, seed=4)
    r, s = StepRunner8(wl), StepRunner8(wl, keep_gradients=False)
    for _ in range(2):
        r.step()
        s.step()
        torch.cuda.synchronize()
        for a, b in zip([r.loss, r.row_loss, r.dHL, r.dW_pred, r.db_pred] + r.dWs + r.dWn + r.db + r.dH[1:2],
                        [s.loss, s.row_loss, s.dHL, s.dW_pred, s.db_pred] + s.dWs + s.dWn + s.db + s.dH[1:2]):
            assert torch.equal(a, b)
        for w in (r, s):
            w.H0.mul_(0.75)


def test_memory_beside_the_float32_step():
    """Per vertex, six layers of 2 x 64 columns: the float32 step keeps 4 (2 x 128) bytes a layer (A H and the
    output) and dH, the 8-bit step 2 x 128; the buffers that all layers share are a few rows of 128 each."""
    n = 20000
    wl = synth.custom(n, "er", 4, [(128, 64)] * 6, head="ce", classes=50, seed=6)

    def used(make):
        before = torch.cuda.memory_allocated()
        r = make()
        r.step()
        torch.cuda.synchronize()
        return (torch.cuda.memory_allocated() - before) / n

    torch.cuda.synchronize()
    plain, kept, shared = used(lambda: StepRunner(wl)), used(lambda: StepRunner8(wl)), used(
        lambda: StepRunner8(wl, keep_gradients=False))
    # beyond one set, a layer keeps dH (4 128) and the rows dZs8, dZn8 (128 each: whole blocks) and Z8 (128)
    assert kept - shared >= 4 * (4 * 128 + 3 * 128 - 16)
    assert shared < 0.75 * plain


def np64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def rounding8(x, rows=1):
    """How far 8-bit values of x may be off it: half a step, 2^-4 of the value, or where that is below the format's
    smallest value up to the whole of that one, 2^-9 of the block's scale, which is below 2^-7 / 1.75 of the block's
    largest magnitude (448 = 1.75 2^8 holds at least half of the range)."""
    n, f = x.shape
    top = np.pad(np.abs(x), ((0, -n % rows), (0, -f % 128))).reshape(-(-n // rows), rows, -1, 128).max((1, 3))
    top = np.repeat(np.repeat(top, rows, 0), 128, 1)[:n, :f]
    return 2.0 ** -4 * np.abs(x) + 2.0 ** -16 / 1.75 * top


def test_input_gradients_against_unrounded_ones():
    """dH of every layer against [dZs || A^T dZn] [Ws || Wn]^T in float64 from dZ before it is rounded: what the two
    roundings of dZ and that of the weights may add up to, element by element, and the float32 sums'."""
    n = 400
    wl = workload()
    r = StepRunner8(wl)
    r.step()
    torch.cuda.synchronize()
    AT = torch.sparse_csr_tensor(r.AT.indptr.long(), r.AT.indices.long(), r.AT.vals.double(), (n, n)).to_dense().cpu().numpy()
    for li in range(r.L - 1, 0, -1):
        fi, h = r.dims[li]
        dY = np64(r.dHL if li == r.L - 1 else r.dH[li + 1].to(torch.bfloat16))
        q = (r.Y8 if li == r.L - 1 else r.X8[li + 1]).values.view(torch.uint8).cpu().numpy()
        z = np.where((q >= 1) & (q <= 126), dY, 0.0)
        W = np64(r.Wb[li])
        e = np.concatenate([rounding8(z[:, :h]), np.abs(AT) @ rounding8(z[:, h:])], 1)
        Z = np.concatenate([z[:, :h], AT @ z[:, h:]], 1)
        mag = np.concatenate([np.abs(z[:, :h]), np.abs(AT) @ np.abs(z[:, h:])], 1)
        e = e + n * 2.0 ** -23 * mag
        e = e + rounding8(np.abs(Z) + e)
        tol = e @ np.abs(W).T + (np.abs(Z) + e) @ rounding8(W, 128).T
        tol += (2 * h + 2) * 2.0 ** -22 * (mag @ np.abs(W).T) + 1e-37
        err = np.abs(np64(r.dH[li]) - Z @ W.T)
        assert np.all(err <= tol), float(np.max(err / tol))
        # a rounding's root mean square is 2^-4 / sqrt(3) of its value at most; three independent ones, and terms of
        # independent signs (the weights are random): 2^-4 in the 2-norm
        assert np.linalg.norm(err) <= 2.0 ** -4 * np.linalg.norm(Z @ W.T), np.linalg.norm(err) / np.linalg.norm(Z @ W.T)
