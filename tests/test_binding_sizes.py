"""Sizes and strides that the library's 32-bit arguments cannot hold, on the
CPU: tensors without memory that say they are on a device."""
import pytest
import torch

from paper_1810_11899_amd import binding as B

FAR = 2 ** 32 + 256          # cut to 32 bits: 256


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def strided(shape, stride, dtype=torch.float32):
    return torch.empty_strided(shape, stride, dtype=dtype, device="meta").as_subclass(OnDevice)


class Space:
    """Stands for a Workspace."""

    def get(self, nbytes):
        return strided((256,), (1,), torch.uint8)


@pytest.fixture(autouse=True)
def no_calls(monkeypatch):
    """No call of the library is made."""
    monkeypatch.setattr(B, "_launch", lambda where, *args: pytest.fail(f"{where} was called"))


def rows4(n, f):
    return B.Rows4.of(strided((n, -(-f // 256) * 128), (-(-f // 256) * 128, 1), torch.uint8),
                      strided((-(-f // 256), -(-n // 64), 512), (-(-n // 64) * 512, 512, 1), torch.uint8), f)


@pytest.mark.parametrize("shape, stride", [((2, 256), (FAR, 1)), ((2, 256), (2 ** 31, 1)), ((FAR, 1), (1, 1)),
                                           ((1, FAR), (FAR, 1))])
def test_rows_of_a_tensor(shape, stride):
    with pytest.raises(ValueError, match="32 bits"):
        B._ld(strided(shape, stride))


def test_the_largest_that_fit():
    assert B._ld(strided((2, 256), (2 ** 31 - 1, 1))) == 2 ** 31 - 1
    assert B._ld(strided((2 ** 31 - 1, 1), (1, 1))) == 1
    assert B._ld(strided((1, 256), (FAR, 1))) >= 256          # (one row of a far larger array)


def test_rows_in_4_bits():
    piece = strided((1, 1, 512), (512, 512, 1), torch.uint8)
    with pytest.raises(ValueError, match="32 bits"):
        B.Rows4.of(strided((2, 128), (FAR, 1), torch.uint8), piece, 256)
    with pytest.raises(ValueError, match="32 bits"):
        B.Rows4.of(strided((FAR, 128), (128, 1), torch.uint8),
                   strided((1, FAR // 64, 512), (FAR * 8, 512, 1), torch.uint8), 256)
    with pytest.raises(ValueError, match="32 bits"):
        B.Rows4.of(strided((1, FAR // 2), (FAR // 2, 1), torch.uint8),
                   strided((FAR // 256, 1, 512), (512, 512, 1), torch.uint8), FAR)


def test_rows_in_8_bits():
    values = strided((2, 128), (FAR, 1), torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="32 bits"):
        B.Rows8.of(values, strided((2, 1), (1, 1), torch.uint8))
    with pytest.raises(ValueError, match="32 bits"):
        B.Rows8.of(strided((FAR, 128), (128, 1), torch.float8_e4m3fn), strided((FAR, 1), (1, 1), torch.uint8))


def test_calls_of_the_4_bit_rows():
    far, near = strided((2, 256), (FAR, 1)), strided((2, 256), (256, 1))
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_rows4_pack(far, Space(), out=rows4(2, 256))
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_rows4_pack(near, Space(), out=rows4(2, 256), mask=far)
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_rows4_unpack(rows4(2, 256), far)
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_rows4_product(rows4(2, 40), rows4(256, 40), far, Space())


def test_calls_of_the_orthogonalised_update():
    far, near = strided((2, 256), (FAR, 1)), strided((2, 256), (256, 1))
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_orthogonalise(far, near, Space())
    with pytest.raises(ValueError, match="32 bits"):
        B.gcn_orthogonalise(near, far, Space())
    for k in range(3):
        with pytest.raises(ValueError, match="32 bits"):
            B.MuonStep(*([far if i == k else near] for i in range(3)))
