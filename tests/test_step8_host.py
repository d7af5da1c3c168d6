"""The 8-bit step's handling of devices and buffers, on the CPU."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_1810_11899_amd import runner
from paper_1810_11899_amd.runner import StepRunner8


@pytest.mark.parametrize("method", ["forward", "head", "backward", "step"])
def test_every_call_of_a_step_is_made_on_the_buffers_device(monkeypatch, method):
    """Calls without a stream go to the current device's: with another device current the aggregations would run
    there, beside the products on the buffers' device."""
    current, calls = [0], []

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d.index
        yield
        current[0] = before

    def call(*args, **kwargs):
        calls.append(current[0])
        return torch.zeros(4, 16)

    monkeypatch.setattr(torch.cuda, "device", device)
    for name in ("gcn_weights8_pack", "gcn_rows8_pack", "gcn_rows8_unpack", "gcn_rows8_product", "gcn_rows8_weight_grad",
                 "gcn_aggregate", "gcn_class_loss", "gcn_csr_transpose_symmetric", "gcn_csr_transpose_into"):
        monkeypatch.setattr(runner.B, name, call)
    r = StepRunner8.__new__(StepRunner8)
    part = lambda *s: torch.zeros(s)
    rows = SimpleNamespace(values=part(4, 16))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    r.__dict__.update(
        L=2, dims=[(8, 8), (16, 8)], H0=SimpleNamespace(device=torch.device("cuda", 1)), A=SimpleNamespace(),
        AT=SimpleNamespace(vals=None, indptr=None, indices=None), symmetric=True, ws=None,
        W=[(part(8, 8), part(8, 8), part(16))] * 2, Wb=[part(8, 16)] * 2, W8=[(None, None, rows)] * 2, X8=[rows] * 2,
        G8=[rows] * 2, Y8=rows, Z8=[rows] * 2, dZs8=[rows] * 2, dZn8=[rows] * 2, _wide=part(4, 16), _low=[part(4, 16)] * 2,
        HL=part(4, 16), dHL=part(4, 16), W_pred=None, b_pred=None, labels=None, loss=None, row_loss=None, dW_pred=None,
        db_pred=None, dWs=[None] * 2, dWn=[None] * 2, db=[part(16)] * 2, dH=[part(4, 16)] * 2)
    getattr(r, method)()
    assert calls and set(calls) == {1} and current == [0]
