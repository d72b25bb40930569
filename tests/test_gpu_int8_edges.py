"""8-bit integer weights at the ends of what the calls take: the longest rows, more rows than one launch holds.  A row's
bits do not depend on the other rows of a call, so large calls are held against small ones."""
import math

import pytest
import torch

from paper_2605_23296_amd import binding as B
from tests.test_gpu_int8 import RULES, by_products, check_route, codes, experts, gen, in_form, layer, product, routed, rows_of, scales

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


def same_as_tiles(M, N, K, epilogue, dtype="bf16", res=False):
    """The call's product and the one in 64 x 64 tiles: integer sums, the same bits."""
    lay = layer(dtype=dtype)
    a, b, sa, sb = codes(M, K, 1, -128), codes((1 + epilogue) * N, K, 2, -128), scales(M, 3), scales((1 + epilogue) * N, 4) / math.sqrt(K) / 5000
    r = rows_of(M, N, dtype, 5) if res else None
    assert torch.equal(product(lay, a, sa, b, sb, r, epilogue, ws=False), in_form(lay, 5, a, sa, b, sb, r, epilogue)), (M, N, K)


# The weight stream has a kernel, with its own ring, for 1 to 8 column tiles of 16 (SwiGLU: 8) a workgroup, as many as one workgroup per compute unit
# of 256 needs, and for 1 .. 8 and 9 .. 16 rows.  K: 1, 3, 16, 18, 32, 50 and 64 units of 128, dealt to 16 wavefronts, the last one whole or cut.
@pytest.mark.parametrize("epilogue", [0, 1])
@pytest.mark.parametrize("tiles", range(1, 9))
def test_weight_streams_of_every_width(tiles, epilogue):
    N = (8 if epilogue else 16) * 256 * (tiles - 1) + 24
    for M in (1, 8, 9, 16):
        for K in (16, 128, 272, 2048, 2192, 4080, 6288, 8192):
            same_as_tiles(M, N, K, epilogue, res=epilogue == 0 and M in (8, 9))
    same_as_tiles(5, N, 2192, epilogue, "fp32", res=epilogue == 0)
    same_as_tiles(13, N, 2192, epilogue, "fp32", res=epilogue == 0)


# Beyond one round of workgroups: as few rounds as 8 column tiles a workgroup allow
@pytest.mark.parametrize("M", [4, 12])
@pytest.mark.parametrize("N,epilogue", [(16 * 256 * 8 + 8, 0), (16 * 256 * 11 + 3, 0), (8 * 256 * 8 + 40, 1), (8 * 256 * 15, 1)])
def test_weight_streams_in_rounds(M, N, epilogue):
    same_as_tiles(M, N, 1040, epilogue)


# 17 .. 32 and 33 .. 48 rows, one and two column tiles a workgroup of 8 wavefronts: sizes that the call streams
@pytest.mark.parametrize("M,tiles,K", [(M, 1, K) for M in (17, 32, 33, 48) for K in (16, 144, 1024, 1168, 2064, 3968)] +
                         [(M, 2, K) for M in (17, 32) for K in (16, 144, 1024, 1168, 2064, 3968, 4096, 6288, 8192)] +
                         [(M, 2, K) for M in (33, 48) for K in (4096, 4112, 5136, 6144)])
def test_weight_streams_of_more_rows(M, tiles, K):
    for epilogue in (0, 1):
        N = (8 if epilogue else 16) * 256 * (tiles - 1) + 24
        same_as_tiles(M, N, K, epilogue, res=epilogue == 0)
    same_as_tiles(M, 4096 * (tiles - 1) + 24, K, 0, "fp32")


# 2^21 rows of a launch; gate: one row for all or a row each
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gate", ["vector", "apart"])
def test_norms_and_codes_of_more_rows_than_one_launch_has(dtype, gate):
    rows, d = 2 ** 21 + 5, 64
    lay, x, b = layer(d=d, dtype=dtype), rows_of(rows, d, dtype, 1), rows_of(rows, d, dtype, 3)
    g_post, g_pre = rows_of(1, d, dtype, 5)[0], rows_of(1, d, dtype, 7)[0]
    wide = rows_of(rows, d + 8, dtype, 9)
    g = wide[0, :d].contiguous() if gate == "vector" else wide[:, :d]

    def norm(at):
        part = lambda t: t[at] if t.dim() > 1 else t   # noqa: E731
        n = len(x[at])
        out = [torch.full((n + 1, d), 7.0, dtype=x.dtype, device="cuda"), torch.full((n + 1, d), 7.0, dtype=x.dtype, device="cuda"),
               torch.full((n + 1, d), 7, dtype=torch.int8, device="cuda"), torch.full((n + 1,), 7.0, device="cuda")]
        h, m, q, s = (t[:n] for t in out)
        lay.compact_block_norm(part(x), b=part(b), g_post=g_post, gate=part(g), alpha=0.7, h=h, g_pre=g_pre, n=m, q=q, q_scale=s)
        assert all(bool((t[n] == 7).all()) for t in out)
        return h, m, q, s

    def row_codes(at):
        n = len(x[at])
        q, s = torch.full((n + 1, d), 7, dtype=torch.int8, device="cuda"), torch.full((n + 1,), 7.0, device="cuda")
        lay.compact_quant_i8(wide[at, :d], q[:n], s[:n])
        assert bool((q[n] == 7).all()) and float(s[n]) == 7.0
        return q[:n], s[:n]
    for call in (norm, row_codes):
        full = call(slice(0, rows))
        for at in pieces(rows, 2 ** 20, 2 ** 21):
            assert all(torch.equal(f[at], small) for f, small in zip(full, call(at)))


# 2^25 rows of a launch
@pytest.mark.parametrize("rule", [dict(score="softmax"), dict(score="sigmoid", n_groups=4, topk_groups=2, group_top=2)])
def test_routing_of_more_rows_than_one_launch_has(rule):
    rows, E, k = 2 ** 25 + 3, 8, 2
    lay, rule = layer(E=E, k=k), B.RouteRule(**rule)
    x = torch.randn((rows, E), generator=gen(1), device="cuda")
    bias = 0.1 * torch.randn(E, generator=gen(2), device="cuda")

    def choose(at):
        logits = x[at]
        idx, w = torch.full((len(logits) + 1, k), -7, dtype=torch.int32, device="cuda"), torch.full((len(logits) + 1, k), -7.0, device="cuda")
        lay.compact_route(rule, logits, bias, idx[:-1], w[:-1])
        assert bool((idx[-1] == -7).all()) and bool((w[-1] == -7.0).all())
        return idx[:-1], w[:-1]
    full = choose(slice(0, rows))
    for at in pieces(rows, 2 ** 24, 2 ** 25):
        assert all(torch.equal(f[at], small) for f, small in zip(full, choose(at)))


HARD = {"coarse": lambda x: torch.round(x * 2) / 2, "alike": lambda x: torch.where(x > 1.0, 1.0, -1.0), "close": lambda x: 1 + x * 2.0 ** -21, "low": lambda x: x * 3 - 100,
        "tiny": lambda x: x * 1e-30, "masked": lambda x: x.index_fill(1, torch.arange(0, x.shape[1], 3), -math.inf), "large": lambda x: x * 20}


@pytest.mark.parametrize("kind", HARD)
@pytest.mark.parametrize("E", [64, 256])
@pytest.mark.parametrize("bias", [False, True])
def test_routing_of_hard_rows_by_kind(kind, E, bias):
    """Rows that 32 bits do not decide, kind by kind, so that how many of each rest on numbers closer than 2^-40 is known: of scores that differ from 1
    by less than that (large) any number do, of close scores whose sums rank groups some half, of the other kinds hardly one."""
    x = HARD[kind](torch.randn((400, E), generator=torch.Generator().manual_seed(3)))
    b = torch.round(8 * torch.randn(E, generator=torch.Generator().manual_seed(4))) / 64 if bias else None
    for rule in RULES[:6]:
        sums = rule.get("group_top") == 2 and not bias
        check_route(layer(E=E, k=8), rule, x.cuda(), None if b is None else b.cuda(), share=-1 if kind == "large" else 0.3 if kind == "close" and sums else 0.97)
