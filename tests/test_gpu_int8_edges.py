"""8-bit integer weights at the ends of what the calls take: the longest rows, more rows than one launch holds.  A row's
bits do not depend on the other rows of a call, so large calls are held against small ones."""
import pytest
import torch

from tests.test_gpu_int8 import by_products, codes, experts, layer, product, routed, rows_of, scales

pytestmark = pytest.mark.gpu


def pieces(n, *borders, k=20):
    """Some rows at either end and around the borders between launches."""
    return [slice(max(0, b - k), min(n, b + k)) for b in (0, *borders, n)]


@pytest.mark.parametrize("cols", [2 ** 31 - 1023, 2 ** 31 - 1])
def test_codes_of_the_longest_rows(cols):
    """The column that is looked at next passes 2^31 for the first time, and at its most."""
    x, room = torch.zeros((1, cols), dtype=torch.bfloat16, device="cuda"), 4096
    buf, scale = torch.full((cols + room,), 77, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    at, value = [0, 1023, 2 ** 30 + 5, cols - 1025, cols - 2, cols - 1], [127.0, -3.0, 12.0, -127.0, 5.0, -64.0]
    x[0, at] = torch.tensor(value, dtype=torch.bfloat16, device="cuda")
    layer().compact_quant_i8(x, buf[:cols].view(1, cols), scale)
    assert bool((buf[cols:] == 77).all()) and float(scale) == 1.0
    assert buf[at].tolist() == value
    buf[at] = 0
    assert not any(bool(part.any()) for part in buf[:cols].split(2 ** 28))


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


def test_experts_whose_products_need_more_workgroups_than_one_launch_has():
    E, k, d, F, rows = 8, 1, 64, 131008, 270_000
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5)
    need = lay.moe_ffn_i8_workspace_bytes(rows)
    assert need == lay.moe_ffn_i8_workspace_bytes(2 * rows)     # of a piece
    lay.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lay.compact_moe_ffn_i8(ex, m, ms, h, idx, w, y[:rows])
    lay.ws = None
    assert bool((y[rows] == 7.0).all())
    border = next(n for n in range(rows) if lay.moe_ffn_i8_workspace_bytes(n) == need)
    for part in pieces(rows, border):
        assert torch.equal(y[:rows][part], by_products(E, d, F, ex, *(t[part].contiguous() for t in (m, ms, h, idx, w))))


def test_products_of_more_rows_than_one_launch_of_workgroups():
    lay, M, K, N = layer(), 2 ** 30 + 200, 16, 1
    a, b, sa, sb = codes(M, K, 1), codes(N, K, 2), scales(M, 3), scales(N, 4) / 5000
    r = scales(M, 5)[:, None].bfloat16()
    for res in (None, r):
        c = product(lay, a, sa, b, sb, res)
        for at in pieces(M, 2 ** 30 - 256, 2 ** 30 - 128, 2 ** 30):
            assert torch.equal(c[at], product(lay, a[at].contiguous(), sa[at].contiguous(), b, sb, None if res is None else res[at].contiguous()))
        del c
