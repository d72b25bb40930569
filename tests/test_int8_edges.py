"""8-bit integer weights on the host: the ends of what the calls take."""
import ctypes as C

import pytest

from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS, LayerConfig
from tests.test_int8 import P, code


@pytest.mark.parametrize("epilogue,most", [(0, 2 ** 29 - 128), (1, 2 ** 28 - 64)])
def test_columns_of_a_product_are_bounded_alike_by_the_call_and_its_workspace(epilogue, most):
    lay, n = B.Layer(WORKLOADS["dense_8x4096"].layer, None), C.c_size_t()
    for rows in (1, 16, 64, 2 ** 31 - 1):
        assert code(lay, "compact_gemm_i8_workspace_bytes", rows, most, 16, epilogue, C.byref(n)) == 0
        assert code(lay, "compact_gemm_i8_workspace_bytes", rows, most + 1, 16, epilogue, C.byref(n)) == 2
        assert code(lay, "compact_gemm_i8", P, P, P, P, None, P, rows, most + 1, 16, epilogue, None, 0, None) == 2


@pytest.mark.parametrize("d,F,k", [(2880, 2880, 4), (64, 131008, 8), (8192, 4096, 1)])
def test_experts_of_the_most_rows_fit_a_card(d, F, k):
    """2^26 / top_k rows, as many as the call takes, run in a workspace that a card of 288 GB holds, which grows with the rows up to there."""
    lay = B.Layer(LayerConfig(d_model=d, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=F, n_experts=128, top_k=k, dtype="bf16"), None)
    need = [lay.moe_ffn_i8_workspace_bytes(2 ** n) for n in range(24)] + [lay.moe_ffn_i8_workspace_bytes(2 ** 26 // k)]
    assert need == sorted(need) and need[8] < need[10] < need[12] and need[-1] < 200e9
