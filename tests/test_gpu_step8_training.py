"""The 8-bit step as a training loop runs it: weights that change between the
steps."""
import pytest
import torch

from tests.gpu_util import require_gpu
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
