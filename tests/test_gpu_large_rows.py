"""Calls of more rows than one launch of workgroups can hold (2^32 threads): the rows at either end and around the borders between launches have
the bits of small calls."""
import pytest
import torch

from tests.test_gpu_int8 import layer, rows_of
from tests.test_gpu_int8_edges import pieces

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rmsnorm(dtype):
    rows, d = 2 ** 24 + 5, 64
    lay, x = layer(d=d, dtype=dtype), rows_of(rows, d, dtype, 1)
    g, y = rows_of(1, d, dtype, 2)[0], torch.full((rows + 1, d), 7.0, dtype=x.dtype, device="cuda")
    lay.compact_rmsnorm(x, g, y[:rows])
    assert bool((y[rows] == 7.0).all())
    for at in pieces(rows, 2 ** 23, 2 ** 24):
        small = torch.empty_like(y[:rows][at])
        lay.compact_rmsnorm(x[at].contiguous(), g, small)
        assert torch.equal(y[:rows][at], small)
