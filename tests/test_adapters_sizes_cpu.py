"""Sizes at which the calls for many adapters leave the fast kernels, as the workspace's size tells."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import build
    build.build()
    from paper_2407_17029_b200 import binding
    return binding


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("P,Q,l1,l2", [(1, 8, 1 << 22, 8), (1, 8, 8, 1 << 22), (3, 8, 1 << 29, 8), (8, 8, 8, 1 << 27), (1, 8, 2 ** 31 - 8, 8)])
def test_lambdas_of_which_a_tile_passes_31_bits(qb, P, Q, l1, l2, backward):
    # 128 columns of q are 128 lambda numbers of a row, whose bytes the kernel counts in 32 bits: the general path's workspace alone
    r, T = 8, 5
    size = lambda l1, l2: qb._lib.qblora_adapters_workspace_bytes(  # noqa: E731
        ctypes.byref(qb._CAdapterBank(P * l1, Q * l2, l1, l2, 2, r, None, None, None, None)), T, backward)
    general = 256 + 4 * T * ((P + r) + (Q + r) * backward)
    general = (general + 255) // 256 * 256
    assert size(l1, l2) == general < size(8, 8)
    assert size((1 << 22) - 8, 8) == size(8, (1 << 22) - 8) == size(8, 8)            # the largest that stay
