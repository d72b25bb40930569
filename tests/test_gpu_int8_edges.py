"""8-bit integer weights at the ends of what the calls take: the longest rows, more rows than one launch holds.  A row's
bits do not depend on the other rows of a call, so large calls are held against small ones."""
import pytest
import torch

from tests.test_gpu_int8 import by_products, codes, experts, layer, routed, rows_of, scales

pytestmark = pytest.mark.gpu


def pieces(n, *borders, k=20):
    """Some rows at either end and around the borders between launches."""
    return [slice(max(0, b - k), min(n, b + k)) for b in (0, *borders, n)]


def test_experts_of_more_rows_than_one_launch_of_workgroups():
    E, k, d, F, rows = 8, 1, 64, 64, 2 ** 24 + 5
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5)
    lay.ws = torch.empty(lay.moe_ffn_i8_workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lay.compact_moe_ffn_i8(ex, m, ms, h, idx, w, y[:rows])
    assert bool((y[rows] == 7.0).all())
    for at in pieces(rows, 2 ** 23, 2 ** 24 - 1):
        assert torch.equal(y[:rows][at], by_products(E, d, F, ex, *(t[at].contiguous() for t in (m, ms, h, idx, w))))
