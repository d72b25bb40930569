"""Paged cache in 8 bits, on the host: its definition at the top of the range, and what its calls refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged8 as P8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS
from tests.test_paged import _kv, _step


@pytest.mark.parametrize("big", [float(torch.finfo(torch.bfloat16).max), float(torch.finfo(torch.float32).max), 248 * 2.0 ** 120, 241 * 2.0 ** 120])
def test_the_largest_finite_values_are_cached_as_finite_ones(big):
    p = P8.Pages(1, 16, 1, 4)
    row = np.array([big, -big, 240 * 2.0 ** 120, 2.0 ** 127]).reshape(1, 1, 4)
    p.write([0], row, -row)
    assert p.scale["k"][0, 0] == p.scale["v"][0, 0] == 247
    top = 240 * 2.0 ** 120
    assert p.rows("k", [0], 1).ravel().tolist() == [top, -top, top, 2.0 ** 127]
    assert p.rows("v", [0], 1).ravel().tolist() == [-top, top, -top, -2.0 ** 127]
    assert np.isfinite(p.rows("k", [0], 1).astype(np.float32)).all()
    # a page that such a row joins late is rounded to its scale, in range
    p = P8.Pages(1, 16, 1, 4)
    p.write([0], row * 0 + 448 * 2.0 ** 119, row)
    p.write([1], row, row)
    assert p.rows("k", [0], 1).ravel().tolist() == [448 * 2.0 ** 119] * 4


def test_a_plan_takes_no_more_rows_than_its_threads_can_count():
    lay = B.Layer(WORKLOADS["dense_8x4096"].layer, None)
    for rows in (1 << 30, 1 << 29, (1 << 26) + 1):
        assert lay.L.compact_paged_plan(lay.ctx, C.byref(_kv()), C.byref(_step(max_rows=rows)), None) == 2, rows
