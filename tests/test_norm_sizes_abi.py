"""The longest tensors that the norm of a reduction takes: decided on the host, before alignment is looked at and anything is launched."""
import ctypes

import pytest

from paper_2506_17615_amd import binding as eq
from test_norm_abi import lib                                            # noqa: F401  (the fixture)
from test_serving_abi import ALIGN, SHAPE


@pytest.mark.parametrize("rows,cols,status", ((1 << 25, 1 << 15, ALIGN), ((1 << 25) + 1, 1 << 15, SHAPE), ((1 << 31) - 1, 1 << 15, SHAPE),
                                              ((1 << 31) - 1, 512, ALIGN), ((1 << 31) - 1, 544, SHAPE)))
def test_partials_of_up_to_2_to_the_40(lib, rows, cols, status):         # noqa: F811
    """Addresses far from each other, that nothing reads; the partial's is odd."""
    outputs = eq._CNormOutputs(codes=1 << 50, scales=1 << 51, block=32)
    partials = (ctypes.c_void_p * 1)((1 << 48) + 8)
    assert lib.equarx_norm_reduced(partials, 1, 32, None, 0, None, rows, cols, 1e-6, 0, ctypes.byref(outputs), None) == status
