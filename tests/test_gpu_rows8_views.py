"""Views that the calls on 8-bit rows refuse, and those next to them that they take."""
import numpy as np
import pytest
import torch

from tests.gpu_util import require_gpu
from paper_1810_11899_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def e4m3(*shape):
    """Positive 8-bit values: a mask that keeps everything."""
    return torch.full(shape, 0x38, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)


def test_weight_grad_refuses_a_mask_whose_rows_share_memory():
    n, f, N = 300, 64, 40
    X8 = B.gcn_rows8_pack(torch.ones((n, f), device="cuda"), B.Rows8(n, f))
    dY, dW, ws = torch.ones((n, N), device="cuda"), torch.full((f, N), 5.0, device="cuda"), B.Workspace()
    for mask in (e4m3(1, N).expand(n, N), torch.as_strided(e4m3(n + N), (n, N), (1, 1)),
                 torch.as_strided(e4m3(n * N), (n, N), (N - 1, 1))):
        with pytest.raises(B.GcnError):
            B.gcn_rows8_weight_grad(X8, dY, dW, ws, mask=mask)
    torch.cuda.synchronize()
    assert float(dW.min()) == 5.0
    B.gcn_rows8_weight_grad(X8, dY, dW, ws, mask=e4m3(n, N))
    assert np.all(dW.cpu().numpy() == n)
    one = B.gcn_rows8_pack(torch.ones((1, f), device="cuda"), B.Rows8(1, f))
    B.gcn_rows8_weight_grad(one, dY[:1], dW, ws, mask=e4m3(1, N).expand(1, N))
    assert np.all(dW.cpu().numpy() == 1.0)


def test_rows_of_whole_blocks_only():
    buf = torch.zeros((8, 304), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scale = torch.zeros((8, 1), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        B.Rows8.of(buf[:, 192:292], scale)
    r = B.Rows8.of(buf[:, 176:276], scale)     # the last row's block ends with the buffer
    B.gcn_rows8_pack(torch.ones((8, 100), device="cuda"), r)
    assert np.all(B.gcn_rows8_unpack(r, torch.empty((8, 100), device="cuda")).cpu().numpy() == 1.0)
