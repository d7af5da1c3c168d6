"""Sizes and addresses that the 8-bit rows and the many-class loss refuse, on
the CPU: every refusal comes before a launch."""
import ctypes
import os

import pytest

from paper_1810_11899_amd import binding as B
from paper_1810_11899_amd import build as pkg_build

P = ctypes.c_void_p
FAKE = P(0x10000)
MOST = 0x7FFFFE00


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pkg_build.LIB_PATH):
        pkg_build.build_library()
    return B.lib()


@pytest.mark.parametrize("n, f, N", [(10, MOST + 1, 64), (10, 2 ** 31 - 1, 64), (10, 64, MOST + 1), (10, 64, 2 ** 31 - 1),
                                     (MOST + 1, 64, 64)])
def test_weight_grad_workspace_of_sizes_that_the_call_refuses(L, n, f, N):
    """0, not the result of an overflow."""
    assert L.gcn_rows8_weight_grad_workspace_bytes(n, f, N) == 0
    assert L.gcn_rows8_weight_grad_workspace_bytes(min(n, MOST), min(f, MOST), min(N, MOST)) > 0
