"""Calls of more rows than one launch of workgroups can hold (2^32 threads): the rows at either end and around the borders between launches have
the bits of small calls."""
import pytest
import torch

from paper_2605_23296_amd import binding as B
from tests.test_gpu_int8 import gen, layer, rows_of
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


def test_routing_by_the_layers_own_rule():
    rows, d, E, k = 2 ** 26 + 5, 64, 8, 2
    lay, m = layer(d=d, E=E, k=k), torch.randn((rows, d), generator=gen(1), device="cuda", dtype=torch.bfloat16)
    wr = torch.randn((E, d), generator=gen(2), device="cuda").bfloat16()
    out = lambda n: (torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.full((n, k), -7.0, device="cuda"), torch.empty((n, E), device="cuda"))   # noqa: E731
    full = out(rows)
    lay.compact_moe_route(m, wr, *full)
    for at in pieces(rows, 2 ** 25, 2 ** 26):
        small = out(len(m[at]))
        lay.compact_moe_route(m[at].contiguous(), wr, *small)
        assert all(torch.equal(f[at], s) for f, s in zip(full, small))


def test_routing_by_a_rule_from_the_rows():
    rows, d, E, k = 2 ** 25 + 3, 64, 8, 2
    lay, m = layer(d=d, E=E, k=k), torch.randn((rows, d), generator=gen(1), device="cuda", dtype=torch.bfloat16)
    wr, bias = torch.randn((E, d), generator=gen(2), device="cuda").bfloat16(), 0.1 * torch.randn(E, generator=gen(3), device="cuda")
    out = lambda n: (torch.empty((n, E), device="cuda"), torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.full((n, k), -7.0, device="cuda"))   # noqa: E731
    for rule in (dict(score="sigmoid", n_groups=4, topk_groups=2, group_top=2), dict(score="softmax")):
        rule, full = B.RouteRule(**rule), out(rows)
        lay.compact_route(rule, full[0], bias, full[1], full[2], m=m, w_router=wr)
        for at in pieces(rows, 2 ** 24, 2 ** 25):
            small = out(len(m[at]))
            lay.compact_route(rule, small[0], bias, small[1], small[2], m=m[at].contiguous(), w_router=wr)
            assert all(torch.equal(f[at], s) for f, s in zip(full, small))
