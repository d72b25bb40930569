"""8-bit integer weights on the host: the ends of what the calls take."""
import ctypes as C

import pytest

from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS
from tests.test_int8 import P, code


@pytest.mark.parametrize("epilogue,most", [(0, 2 ** 29 - 128), (1, 2 ** 28 - 64)])
def test_columns_of_a_product_are_bounded_alike_by_the_call_and_its_workspace(epilogue, most):
    lay, n = B.Layer(WORKLOADS["dense_8x4096"].layer, None), C.c_size_t()
    for rows in (1, 16, 64, 2 ** 31 - 1):
        assert code(lay, "compact_gemm_i8_workspace_bytes", rows, most, 16, epilogue, C.byref(n)) == 0
        assert code(lay, "compact_gemm_i8_workspace_bytes", rows, most + 1, 16, epilogue, C.byref(n)) == 2
        assert code(lay, "compact_gemm_i8", P, P, P, P, None, P, rows, most + 1, 16, epilogue, None, 0, None) == 2
