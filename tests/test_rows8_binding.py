"""What the Python binding makes of the tensors of the 8-bit rows, on the CPU:
tensors that say they are on a device, and the library's call recorded."""
import pytest
import torch

from paper_1810_11899_amd import binding as B


class OnDevice(torch.Tensor):
    """A CPU tensor that the binding takes for one on device 0, or on the device of its `where`."""
    where = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.where


def dev(t, where=0):
    t = t.as_subclass(OnDevice)
    t.where = where
    return t


def rows8(n, f):
    nb = -(-f // 128)
    values = torch.zeros((max(n, 1), nb * 128), dtype=torch.uint8).view(torch.float8_e4m3fn)[:n, :f]
    return B.Rows8.of(dev(values), dev(torch.zeros((n, nb), dtype=torch.uint8)))


class Space:
    """Stands for a Workspace."""
    buf = dev(torch.zeros(8, dtype=torch.uint8))

    def args(self, nbytes):
        return 0x10000, nbytes


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, (name, arguments), which are not made."""
    made = []
    monkeypatch.setattr(B, "_launch", lambda where, device, stream, *args: made.append((where, args)))
    return made


# ---------------------------------------------------------------- the mask's rows
def mask_stride(calls, mask, n, N):
    B.gcn_rows8_weight_grad(rows8(n, 64), dev(torch.zeros(n, N)), dev(torch.zeros(64, N)), Space(), mask=dev(mask))
    return calls[-1][1][2]


def test_mask_rows_that_share_memory_keep_their_stride(calls):
    """The library refuses a row stride below the columns: the binding passes it on as it is."""
    e4m3 = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(torch.float8_e4m3fn)
    n, N = 50, 32
    assert mask_stride(calls, e4m3(1, N).expand(n, N), n, N) == 0
    assert mask_stride(calls, torch.as_strided(e4m3(n + N), (n, N), (1, 1)), n, N) == 1
    assert mask_stride(calls, e4m3(n, N), n, N) == N
    assert mask_stride(calls, e4m3(n, 128)[:, 64:64 + N], n, N) == 128
    assert mask_stride(calls, e4m3(1, N).expand(1, N), 1, N) >= N          # one row: any stride
    assert mask_stride(calls, torch.as_strided(e4m3(N), (1, N), (0, 1)), 1, N) >= N


# ---------------------------------------------------- 8-bit rows kept elsewhere
def kept(rows, cols, where=0):
    return dev(torch.zeros((rows, cols), dtype=torch.uint8).view(torch.float8_e4m3fn), where)


def scale(rows, blocks, where=0):
    return dev(torch.zeros((rows, blocks), dtype=torch.uint8), where)


def test_rows_whose_blocks_end_behind_the_memory_are_refused():
    """100 columns from column 192 on of rows of 304: the last row's block of 128 ends 16 bytes behind the buffer."""
    buf = kept(8, 304)
    with pytest.raises(ValueError, match="whole"):
        B.Rows8.of(buf[:, 192:292], scale(8, 1))
    with pytest.raises(ValueError, match="whole"):
        B.Rows8.of(kept(1, 112)[:, :100], scale(1, 1))
    assert B.Rows8.of(buf[:, 176:276], scale(8, 1)).struct.ldq == 304      # up to the very end
    assert B.Rows8.of(buf[:7, 192:292], scale(7, 1)).struct.ldq == 304     # (the row behind the last holds it)
    assert B.Rows8.of(kept(8, 256)[:0, :200], scale(0, 2)).n == 0


def test_weights_whose_blocks_end_behind_the_memory_are_refused():
    whole, cut = kept(100, 128), kept(100, 112)
    assert B.Weights8.of(whole[:, :100], whole[:, :100], scale(1, 1)).K == 100
    for v, vt in ((cut[:, :100], whole[:, :100]), (whole[:, :100], cut[:, :100])):
        with pytest.raises(ValueError, match="whole"):
            B.Weights8.of(v, vt, scale(1, 1))


def test_parts_on_different_devices_are_refused():
    with pytest.raises(ValueError, match="one device"):
        B.Rows8.of(kept(8, 128), scale(8, 1, where=1))
    for at in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        with pytest.raises(ValueError, match="one device"):
            B.Weights8.of(kept(128, 128, at[0]), kept(128, 128, at[1]), scale(1, 1, at[2]))


# ------------------------------------------------------------------- streams
def test_the_current_stream_without_torchs_undocumented_call(monkeypatch):
    """Every call's stream: the documented one where torch does not give the handle alone."""
    class Current:
        cuda_stream = 0x1234

    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(B, "_raw_stream", None)
    assert B._stream() == 0x1234
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0x5000 + device)
    assert B._stream() == 0x5003
    Current.cuda_stream = 0x77
    assert B._stream(Current) == 0x77
