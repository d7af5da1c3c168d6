"""The 8-bit step as a training loop runs it: weights that change between the
steps."""
import pytest
import torch

from tests.gpu_util import require_gpu
from paper_1810_11899_amd import synth
from paper_1810_11899_amd.runner import StepRunner8

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
