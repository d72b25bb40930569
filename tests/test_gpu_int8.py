"""8-bit integer weights: codes, products, norms around a block, routing and the experts' products, against the definition in 64 bits.

Tolerances count roundings: u = 2^-24 is half a step of fp32, 2^-8 that of bf16.  Codes are whole numbers and have to be equal."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import int8 as I8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import LayerConfig

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": U}


def layer(d=256, F=128, E=0, k=0, dtype="bf16"):
    return B.Layer(LayerConfig(d_model=d, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=F, n_experts=E, top_k=k, dtype=dtype), None)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def f64(t):
    return t.double().cpu().numpy()


def rows_of(n, d, dtype, seed):
    x = torch.randn((n, d), generator=gen(seed), device="cuda") * torch.exp(2 * torch.randn((n, 1), generator=gen(seed + 1), device="cuda"))
    return x.to(DT[dtype])


def codes(n, d, seed, lo=-127, hi=127):
    return torch.randint(lo, hi + 1, (n, d), generator=gen(seed), device="cuda", dtype=torch.int8)


def scales(n, seed):
    return torch.exp(torch.randn(n, generator=gen(seed), device="cuda"))


# ---- rows -> codes -----------------------------------------------------------------------------------------------------------

def quantised(lay, x, room=0):
    q = torch.full((x.shape[0] + room, x.shape[1]), 77, dtype=torch.int8, device="cuda")
    s = torch.full((x.shape[0] + room,), 77.0, device="cuda")
    lay.compact_quant_i8(x, q[:x.shape[0]], s)
    assert bool((q[x.shape[0]:] == 77).all()) and bool((s[x.shape[0]:] == 77).all())
    return q[:x.shape[0]], s[:x.shape[0]]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (2, 64), (5, 200), (4, 1000), (33, 4096), (3, 4104), (2, 14336), (2, 28672), (1, 70001), (700, 72), (0, 64), (4, 512), (3, 520),
                                       (5, 1024), (2, 1032), (3, 2048), (1030, 2056), (2, 2880), (1025, 2880), (2, 3080), (3, 8192), (2, 8200), (2, 16392), (1, 32776), (1, 65536),
                                       (1, 65544)])
def test_codes_of_rows(dtype, rows, cols):
    x = rows_of(rows, cols, dtype, 3)
    if rows:
        x[0, cols // 2] = x[0].abs().max() / 2 if cols > 1 else x[0, 0]     # a tie
    q, s = quantised(layer(dtype=dtype), x, 2)
    rq, rs = I8.row_codes(f64(x))
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)


@pytest.mark.parametrize("dtype", DT)
def test_codes_of_values_at_every_size(dtype):
    tiny, big = torch.finfo(DT[dtype]).smallest_normal, torch.finfo(DT[dtype]).max
    x = rows_of(24, 136, dtype, 5)
    x /= x.abs().amax(-1, keepdim=True)
    sizes = [big, big / 3, 1e30, 1e10, 1e-10, 1e-20, 1e-29, 1.1e-30, 1e-31, 3e-37, 2e-38, tiny]
    for i, v in enumerate(sizes):
        x[i] = (x[i].double() * v).to(DT[dtype])
    x[12] = 0
    x[13], x[13, 40] = 0, -2.5
    x[14, 0], x[15, 135], x[16, 9], x[17, 3], x[17, 4] = math.inf, -math.inf, math.nan, math.nan, math.inf
    x[18] = -1.0
    x[20], x[21] = x[20] * tiny * 2.0 ** -4, x[21] * tiny * 2.0 ** -7      # below the normal numbers
    x[19] = torch.arange(136, device="cuda").to(DT[dtype]) - 60.5 if dtype == "fp32" else x[19]    # ties and neighbours of them
    q, s = quantised(layer(dtype=dtype), x)
    rq, rs = I8.row_codes(f64(x))
    assert np.array_equal(q.cpu().numpy(), rq)
    assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("cols,lo,width", [(64, 0, 192), (64, 8, 200), (61, 3, 67), (1000, 1, 1001)])
def test_codes_of_rows_that_lie_apart(dtype, cols, lo, width):
    wide = rows_of(9, width, dtype, 6)
    lay = layer(dtype=dtype)
    a, b = quantised(lay, wide[:, lo:lo + cols]), quantised(lay, wide[:, lo:lo + cols].contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- products ----------------------------------------------------------------------------------------------------------------

def product(lay, a, sa, b, sb, r=None, epilogue=0, ws=True):
    M, K, N = a.shape[0], a.shape[1], b.shape[0] // (2 if epilogue else 1)
    lay.ws = torch.empty(lay.gemm_i8_workspace_bytes(M, N, K, epilogue), dtype=torch.uint8, device="cuda") if ws else None
    c = torch.full((M + 1, N), 7.0, dtype=lay.torch_dtype, device="cuda")
    lay.compact_gemm_i8(a, sa, b, sb, r, c[:M], epilogue)
    assert bool((c[M] == 7.0).all())       # nothing past the last row
    return c[:M]


def check_product(c, a, sa, b, sb, r, epilogue, dtype):
    """Half a step for the sum's conversion, two for the scales, one for the residual, one for the storage type.  SwiGLU: silu' g / silu is at most
    1 + |g|; exp as exp2(g log2 e) is off by |g| 2^-23 and 2^-22, quotient and product by 3 u, all again as large in fp32 at most.  Below g = -88.72 exp(-g) is beyond
    fp32, and the quotient 0 instead of g exp(g), which is less than 88.72 exp(-88.72) < 2^-121 in size.  With bf16 storage the reciprocal instruction stands
    for the quotient: one unit (2 u) more, and 0 where it would be below 2^-126, the least normal number: g < -126 ln 2 = -87.33, and the
    value less than 87.34 * 2^-126 < 2^-119.5."""
    p = torch.tensor(I8.product(a.cpu().numpy(), f64(sa), b.cpu().numpy(), f64(sb)))
    if epilogue:
        g, u = p.chunk(2, -1)
        ref = torch.tensor(I8.silu(g.numpy())) * u
        tol = ref.abs() * ((1 + g.abs()) * 3 * U + 3 * U + g.abs() * 2.0 ** -23 + 2.0 ** -22 + 3 * U) + torch.where(g < -87.3, u.abs() * (2.0 ** -119.5 if dtype == "bf16" else 2.0 ** -121), 0.0)
        tol += ref.abs() * (2 * U if dtype == "bf16" else 0)
    else:
        ref = p + (0 if r is None else r.double().cpu())
        tol = p.abs() * 3 * U + ref.abs() * U
    tol = 1.01 * tol + ref.abs() * HALF[dtype] + 2.0 ** -133       # (the least bf16 step)
    err = (c.double().cpu() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("epilogue,res", [(0, False), (0, True), (1, False)])
@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (1, 8, 64), (2, 3, 48), (3, 16, 128), (5, 100, 144), (8, 96, 4096), (9, 257, 272), (15, 24, 1040), (16, 64, 2880), (17, 64, 128),
                                   (31, 130, 256), (33, 7, 112), (63, 264, 1152), (64, 128, 512), (65, 72, 384), (127, 40, 640), (129, 520, 896), (200, 1001, 208),
                                   (257, 264, 272), (300, 136, 3968), (513, 72, 1024), (17, 96, 4096), (64, 1000, 4112), (130, 77, 6160), (40, 96, 16400), (18, 520, 8208), (49, 72, 8192),
                                   (48, 1000, 336)])
def test_products(dtype, epilogue, res, M, N, K):
    lay = layer(dtype=dtype)
    a, b = codes(M, K, 1), codes((1 + epilogue) * N, K, 2, -128)
    sa, sb = scales(M, 3), scales(len(b), 4) / math.sqrt(K) / 5000
    r = rows_of(M, N, dtype, 5) if res else None
    c = product(lay, a, sa, b, sb, r, epilogue)
    check_product(c, a, sa, b, sb, r, epilogue, dtype)
    assert torch.equal(product(lay, a, sa, b, sb, r, epilogue, ws=False), c)     # a workspace changes no bit
    if lay.gemm_i8_workspace_bytes(M, N, K, epilogue):
        lay.ws = torch.empty(lay.gemm_i8_workspace_bytes(M, N, K, epilogue) - 1, dtype=torch.uint8, device="cuda")   # one that is too small is none
        small = torch.empty_like(c)
        lay.compact_gemm_i8(a, sa, b, sb, r, small, epilogue)
        assert torch.equal(small, c)
    assert (lay.gemm_i8_workspace_bytes(M, N, K, epilogue) > 0) == (M > 48 and K >= 5120 or M > 16 and K > 16000)


def in_form(lay, form, a, sa, b, sb, r, epilogue, slices=1):
    """The product in one of the tile forms (6: 256 x 256 tiles and their halves, mixed), or in slices of K."""
    M, K, N = a.shape[0], a.shape[1], b.shape[0] // (2 if epilogue else 1)
    c = torch.full((M + 1, N), 7.0, dtype=lay.torch_dtype, device="cuda")
    ptr = lambda t: None if t is None else C.c_void_p(t.data_ptr())   # noqa: E731
    sums = torch.empty(slices * M * len(b), dtype=torch.int32, device="cuda")
    lay.check(lay.L.compact_test_gemm_i8_form(lay.ctx, C.c_int32(form), C.c_int32(slices), ptr(sums), ptr(a), ptr(sa), ptr(b), ptr(sb), ptr(r), ptr(c), C.c_int64(M), C.c_int32(N), C.c_int32(K),
                                              C.c_int32(epilogue), C.c_void_p(torch.cuda.current_stream().cuda_stream)))
    assert bool((c[M] == 7.0).all())
    return c[:M]


# one to seven k-tiles of 128, whole and cut; rows and columns just under, at and over the tile edges
@pytest.mark.parametrize("K", [16, 112, 128, 144, 256, 368, 512, 640, 784, 896])
@pytest.mark.parametrize("epilogue,res", [(0, True), (0, False), (1, False)])
def test_every_tile_form_at_its_edges(K, epilogue, res):
    lay = layer()
    for M, N in [(1, 8), (63, 136), (65, 57), (128, 64), (129, 264), (257, 520), (300, 128), (511, 1000), (700, 259)]:
        a, b, sa, sb = codes(M, K, 1), codes((1 + epilogue) * N, K, 2), scales(M, 3), scales((1 + epilogue) * N, 4) / math.sqrt(K) / 5000
        r = rows_of(M, N, "bf16", 5) if res else None
        want = in_form(lay, 5, a, sa, b, sb, r, epilogue)
        check_product(want, a, sa, b, sb, r, epilogue, "bf16")
        for form in (0, 1, 2, 3, 4, 6):
            assert torch.equal(in_form(lay, form, a, sa, b, sb, r, epilogue), want), (M, N, form)
        for form in (2, 3, 4, 5):
            for slices in {min(n, -(-K // 128)) for n in (2, 3, 5, 7)} - {1}:
                assert torch.equal(in_form(lay, form, a, sa, b, sb, r, epilogue, slices), want), (M, N, form, slices)


@pytest.mark.parametrize("M", [1, 16, 40, 200, 700])
def test_the_largest_sums(M):
    """K at its most, codes at their ends: 2^31 is not reached, and nothing is lost before the conversion to fp32."""
    lay, K = layer(dtype="fp32"), 131056
    a, b = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((24, K), -128, dtype=torch.int8, device="cuda")
    b[1], b[2, ::2] = 127, 127
    a[-1, -1] = 127
    one = torch.ones(max(M, 24), device="cuda")
    c = product(lay, a, one, b, one)
    ref = (a.double() @ b.double().t()).float()
    assert torch.equal(c, ref)


def test_the_bits_of_a_row_do_not_depend_on_the_rows_beside_it():
    for dtype, N, K, epi in (("bf16", 520, 2880, 0), ("fp32", 264, 1088, 0), ("bf16", 200, 1152, 1)):
        lay, M = layer(dtype=dtype), 1400
        a, b, sa, sb = codes(M, K, 1), codes((1 + epi) * N, K, 2), scales(M, 3), scales((1 + epi) * N, 4) * 1e-4
        full = product(lay, a, sa, b, sb, None, epi)
        for n in (1, 7, 16, 17, 33, 64, 65, 100, 128, 250, 300, 512, 700, 1025, 1399):
            assert torch.equal(product(lay, a[M - n:].contiguous(), sa[M - n:].contiguous(), b, sb, None, epi), full[M - n:]), (dtype, n)


def test_broken_scales_stay_in_their_rows_and_columns():
    lay = layer()
    for M in (5, 40, 300):
        a, b, sa, sb = codes(M, 256, 1), codes(72, 256, 2), scales(M, 3), scales(72, 4)
        sa[2], sb[9], sa[3] = math.nan, math.nan, 0.0
        c = product(lay, a, sa, b, sb)
        bad = torch.zeros_like(c, dtype=torch.bool)
        bad[2], bad[:, 9] = True, True
        assert torch.equal(c.isnan(), bad) and bool((c[3][~bad[3]] == 0).all())


def test_the_residual_may_be_the_output():
    lay = layer()
    for M in (3, 20, 40, 50, 400):
        for N in (136, 137):
            a, b, sa, sb, r = codes(M, 320, 1), codes(N, 320, 2), scales(M, 3), scales(N, 4) * 1e-3, rows_of(M, N, "bf16", 5)
            want = product(lay, a, sa, b, sb, r)
            lay.compact_gemm_i8(a, sa, b, sb, r, r)
            assert torch.equal(r, want), (M, N)


# ---- norms around a block ------------------------------------------------------------------------------------------------------

def check_norm(lay, x, b, g_post, gate, alpha, g_pre, dtype):
    """Sums of squares of at most 8192 numbers by lanes and then as a tree: 2^-18; root, quotient, products: below that.  n is compared with the norm of
    the h that was stored, the codes with those of the n that was."""
    eps, slack = lay.layer.rms_eps, 2.0 ** -18
    rows = x.shape[0]
    h, n = torch.empty_like(x) if b is not None else None, torch.empty_like(x)
    q, s = torch.full(x.shape, 99, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    lay.compact_block_norm(x, b=b, g_post=g_post, gate=gate, alpha=alpha, h=h, g_pre=g_pre, n=n, q=q, q_scale=s)
    some = lambda t: None if t is None else f64(t)   # noqa: E731
    stored = f64(x)
    if b is not None:
        ref = I8.residual(f64(x), f64(b), some(g_post), some(gate), alpha, eps)
        branch = np.abs(ref - f64(x))
        assert (np.abs(f64(h) - ref) <= branch * slack + np.abs(ref) * (HALF[dtype] * 1.01 + U)).all()
        stored = f64(h)
    ref = I8.rms_norm(stored, f64(g_pre), eps)
    assert (np.abs(f64(n) - ref) <= np.abs(ref) * (slack + HALF[dtype] * 1.01)).all()
    rq, rs = I8.row_codes(f64(n))
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)
    # the outputs one at a time, and in place, have the same bits
    q2, s2, h2 = torch.empty_like(q), torch.empty_like(s), torch.empty_like(x)
    lay.compact_block_norm(x, b=b, g_post=g_post, gate=gate, alpha=alpha, g_pre=g_pre, q=q2, q_scale=s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)
    if b is not None:
        lay.compact_block_norm(x, b=b, g_post=g_post, gate=gate, alpha=alpha, h=h2)
        assert torch.equal(h, h2)
        y, z = x.clone(), b.clone()
        lay.compact_block_norm(y, b=z, g_post=g_post, gate=gate, alpha=alpha, h=y, g_pre=g_pre, n=z)
        assert torch.equal(y, h) and torch.equal(z, n)
    return h, n


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,d", [(1, 64), (3, 128), (5, 448), (70, 512), (4, 1088), (33, 2048), (2, 2112), (9, 2880), (8, 4096), (3, 6080), (5, 8192), (1100, 256), (7, 576), (6, 1024), (5, 1536), (2, 1600), (3, 2048),
                                    (2, 4160)])
@pytest.mark.parametrize("post,gate", [(False, None), (True, "vector"), (False, "rows"), (True, "apart")])
def test_norms_around_a_block(dtype, rows, d, post, gate):
    lay = layer(d=d, dtype=dtype)
    x, b = rows_of(rows, d, dtype, 1), rows_of(rows, d, dtype, 3)
    gain = lambda seed: (1 + 0.2 * torch.randn(d, generator=gen(seed), device="cuda")).to(DT[dtype])   # noqa: E731
    g = None
    if gate:
        wide = torch.randn((rows, d + 64), generator=gen(7), device="cuda").to(DT[dtype])
        g = wide[0, :d].contiguous() if gate == "vector" else wide[:, :d] if gate == "apart" else wide[:, :d].contiguous()
    check_norm(lay, x, b, gain(5) if post else None, g, 0.37, gain(6), dtype)


@pytest.mark.parametrize("dtype", DT)
def test_a_norm_without_a_block_is_the_layers_own(dtype):
    lay = layer(d=2880, dtype=dtype)
    x, g = rows_of(37, 2880, dtype, 1), (1 + 0.2 * torch.randn(2880, generator=gen(2), device="cuda")).to(DT[dtype])
    check_norm(lay, x, None, None, None, 1.0, g, dtype)
    n, y = torch.empty_like(x), torch.empty_like(x)
    lay.compact_block_norm(x, g_pre=g, n=n)
    lay.compact_rmsnorm(x, g, y)
    # both are within check_norm's bound of the same number (its sum of squares is off by 2^-18 at most, whatever the order)
    assert float((n.double() - y.double()).abs().max() / y.abs().max()) <= 2 * (HALF[dtype] * 1.01 + 2.0 ** -18)


@pytest.mark.parametrize("dtype", DT)
def test_broken_rows_and_rows_of_zeros_stay_where_they_are(dtype):
    lay = layer(d=512, dtype=dtype)
    x, b, g = rows_of(8, 512, dtype, 1), rows_of(8, 512, dtype, 3), torch.ones(512, dtype=DT[dtype], device="cuda")
    x[1, 5], b[2, 500], x[3, 0] = math.nan, math.inf, -math.inf
    x[4], b[4] = 0, 0
    h, n, q, s = torch.empty_like(x), torch.empty_like(x), torch.empty((8, 512), dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
    lay.compact_block_norm(x, b=b, h=h, g_pre=g, n=n, q=q, q_scale=s)
    assert s.isnan().tolist() == [False, True, True, True] + 4 * [False] and not q[1:5].any() and s[4] == 0 and not n[4].any()
    assert bool(n[[0, 5, 6, 7]].isfinite().all()) and int(q[[0, 5, 6, 7]].abs().amax(-1).min()) == 127


# ---- routing -------------------------------------------------------------------------------------------------------------------

def check_route(lay, rule, logits, bias, share=0.999):
    """Rows whose choice rests on numbers closer than 2^-40 of them may choose otherwise; `share` of the rows at least do not."""
    E, k, rows = lay.layer.n_experts, lay.layer.top_k, logits.shape[0]
    idx, w = torch.full((rows + 1, k), -7, dtype=torch.int32, device="cuda"), torch.full((rows + 1, k), -7.0, device="cuda")
    lay.compact_route(B.RouteRule(**rule), logits, bias, idx[:rows], w[:rows])
    assert bool((idx[rows] == -7).all()) and bool((w[rows] == -7).all())
    ref, rw, gap = I8.route(f64(logits), None if bias is None else f64(bias), k, **rule)
    clear = gap > 2.0 ** -40
    assert clear.mean() > share
    got = idx[:rows].cpu().numpy()
    assert np.array_equal(got[clear], ref[clear])
    assert (np.sort(got, -1)[:, 1:] != np.sort(got, -1)[:, :-1]).all() and got.min(initial=0) >= 0 and got.max(initial=0) < E
    # scores to a few units, a sum of 8, a quotient, the factor; below fp32's normal numbers half of their step
    assert (np.abs(f64(w[:rows])[clear] - rw[clear]) <= np.abs(rw[clear]) * 2.0 ** -20 + 2.0 ** -150).all()
    return got, f64(w[:rows])


RULES = [dict(score="softmax"), dict(score="softmax", renorm=False, factor=1.5), dict(score="sigmoid"), dict(score="sigmoid", renorm=False, factor=2.5),
         dict(score="sigmoid", n_groups=8, topk_groups=4, group_top=2), dict(score="softmax", n_groups=4, topk_groups=2, group_top=1),
         dict(score="sigmoid", n_groups=2, topk_groups=1, group_top=2, factor=0.1), dict(score="softmax", n_groups=8, topk_groups=8, group_top=2),
         dict(score="sigmoid", n_groups=16, topk_groups=8, group_top=2), dict(score="softmax", n_groups=16, topk_groups=5, group_top=1)]


@pytest.mark.parametrize("E,k", [(8, 1), (16, 2), (64, 6), (128, 4), (160, 8), (232, 5), (256, 8)])
@pytest.mark.parametrize("rule", range(len(RULES)))
@pytest.mark.parametrize("bias", [False, True])
def test_routing(E, k, rule, bias):
    rule = RULES[rule]
    g = rule.get("n_groups", 1)
    if E // g * rule.get("topk_groups", 1) < k or E % g:
        return
    for rows in (1, 3, 67, 1000 if E == 256 else 130):
        x = 2 * torch.randn((rows, E), generator=gen(rows), device="cuda")
        check_route(layer(E=E, k=k), rule, x, 0.1 * torch.randn(E, generator=gen(9), device="cuda") if bias else None)


def test_routing_with_an_odd_number_of_experts():
    lay = layer(E=21, k=5, dtype="fp32")
    for rule in (dict(score="softmax"), dict(score="sigmoid", n_groups=7, topk_groups=3, group_top=2), dict(score="softmax", n_groups=21, topk_groups=5, group_top=2)):
        check_route(lay, rule, torch.randn((90, 21), generator=gen(1), device="cuda"), torch.randn(21, generator=gen(2), device="cuda") * 0.1)


@pytest.mark.parametrize("rule", RULES[:6])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("E,k", [(64, 8), (256, 8)])
def test_routing_of_rows_that_32_bits_do_not_decide(rule, bias, E, k):
    """Logits on a coarse grid, most experts alike, scores a few 2^-26 apart, groups that tie, logits far below zero: the rows that go to the way in 64 bits
    beside rows that do not."""
    lay, x = layer(E=E, k=k), torch.randn((640, E), generator=gen(3), device="cuda")
    x[0::8] = torch.round(x[0::8] * 2) / 2
    x[1::8] = torch.where(x[1::8] > 1.0, 1.0, -1.0)
    x[2::8] = 1 + x[2::8] * 2.0 ** -21
    x[3::8] = x[3::8] * 3 - 100
    x[4::8] = x[4::8] * 1e-30
    x[5::8, ::3] = -math.inf
    x[6::8] *= 20      # (sigmoids that differ from 1 by less than 2^-40; those and rows of 2::8 whose sums fall together are a quarter at most)
    check_route(lay, rule, x, torch.round(8 * torch.randn(E, generator=gen(4), device="cuda")) / 64 if bias else None, share=0.75)


@pytest.mark.parametrize("rule", [dict(score="softmax"), dict(score="sigmoid"), dict(score="sigmoid", n_groups=4, topk_groups=2, group_top=2),
                                  dict(score="softmax", n_groups=8, topk_groups=3, group_top=1, renorm=False)])
@pytest.mark.parametrize("bias", [False, True])
def test_routing_ties_masks_and_broken_logits(rule, bias):
    E, k, inf, nan = 64, 6, math.inf, math.nan
    lay = layer(E=E, k=k)
    x = torch.randn((40, E), generator=gen(1), device="cuda")
    x[0] = 0.25                                   # all equal
    x[1] = torch.arange(E, device="cuda") % 4     # ties in every group
    x[2] = -inf                                   # a row that is masked out
    x[3], x[3, 17] = -inf, 0.5                    # one expert is left
    x[4, ::2] = -inf
    x[5, :60] = -inf                              # fewer than top_k left
    x[6], x[6, 63] = nan, 1.0
    x[7, 3], x[7, 40], x[7, 41] = inf, inf, -inf
    x[8], x[9] = 300.0, -300.0
    x[10, 5], x[11, 6] = 3e38, -3e38
    b = None
    if bias:
        b = 0.1 * torch.randn(E, generator=gen(2), device="cuda")
        b[20], b[21] = -inf, nan                  # experts that are switched off
        b[30:34] = 0.0
    got, w = check_route(lay, rule, x, b)
    assert not w[2].any() and (w >= 0).all() and (np.isfinite(w)).all()
    if bias:
        rest = [i for i in range(40) if i not in (2, 3, 5, 6)]
        assert not np.isin(got[rest], [20, 21]).any()


@pytest.mark.parametrize("E,k,groups,of", [(16, 4, 8, 4), (24, 5, 12, 4), (64, 6, 8, 3), (256, 8, 8, 4), (160, 8, 16, 5)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20])
def test_routing_where_the_biases_of_a_group_cancel(E, k, groups, of, score, size):
    """The two best of every group are size + s and -size + s': their sum is decided by digits that neither has in 32 bits."""
    S, bias = E // groups, torch.full((E,), -size, device="cuda")
    for g in range(groups):
        bias[g * S + g % S] = size
    x = torch.randn((2000, E), generator=gen(E), device="cuda")
    check_route(layer(E=E, k=k), dict(score=score, n_groups=groups, topk_groups=of, group_top=2), x, bias, share=0.99)


@pytest.mark.parametrize("dtype,E", [("bf16", 128), ("fp32", 24)])
@pytest.mark.parametrize("rows", [1, 16, 300])
def test_routing_from_the_rows(dtype, E, rows):
    lay = layer(d=512, E=E, k=4, dtype=dtype)
    m, wr = torch.randn((rows, 512), generator=gen(1), device="cuda").to(DT[dtype]), (0.05 * torch.randn((E, 512), generator=gen(2), device="cuda")).to(DT[dtype])
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    logits, idx, w = torch.empty((rows, E), **f32), torch.empty((rows, 4), **i32), torch.empty((rows, 4), **f32)
    lay.compact_route(B.RouteRule("softmax", renorm=True), logits, None, idx, w, m=m, w_router=wr)
    # the rule of the layer itself: the same experts from the same logits
    idx2, w2, l2 = torch.empty_like(idx), torch.empty_like(w), torch.empty_like(logits)
    lay.compact_moe_route(m, wr, idx2, w2, l2)
    assert torch.equal(logits, l2) and torch.equal(idx, idx2) and float((w - w2).abs().max()) < 2.0 ** -20


# ---- the experts' products -----------------------------------------------------------------------------------------------------

def experts(E, d, F, seed):
    gu, dn = codes(E * 2 * F, d, seed).view(E, 2 * F, d), codes(E * d, F, seed + 1).view(E, d, F)
    sg, sd = scales(E * 2 * F, seed + 2).view(E, 2 * F) / math.sqrt(d) / 5000, scales(E * d, seed + 3).view(E, d) / math.sqrt(F) / 5000
    return B.ExpertsI8(gu, sg, dn, sd)


def by_products(E, d, F, ex, m, ms, h, idx, w):
    """The experts' products out of calls of their own: the same roundings, hence the same bits."""
    bf, f32 = layer(d=d, F=F), layer(d=d, F=F, dtype="fp32")
    rows, k = idx.shape
    out = torch.zeros((rows, k, d), dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        at = (idx == e).nonzero()
        if not len(at):
            continue
        act = product(bf, m[at[:, 0]], ms[at[:, 0]], ex.gate_up[e], ex.gate_up_scale[e], None, 1)
        q, s = quantised(bf, act)
        out[at[:, 0], at[:, 1]] = (product(f32, q, s, ex.down[e], ex.down_scale[e]) * w[at[:, 0], at[:, 1]][:, None]).bfloat16()
    y = h.float()
    for j in range(k):
        y = y + out[:, j].float()
    return y.bfloat16()


def ffn(lay, ex, m, ms, h, idx, w, exact_ws=True):
    lay.ws = torch.full((lay.moe_ffn_i8_workspace_bytes(m.shape[0]),), 0xA5, dtype=torch.uint8, device="cuda")
    y = torch.empty_like(h)
    lay.compact_moe_ffn_i8(ex, m, ms, h, idx, w, y)
    return y


def routed(rows, E, k, seed, uneven=0.0):
    score = torch.randn((rows, E), generator=gen(seed), device="cuda") + uneven * torch.randn(E, generator=gen(seed + 1), device="cuda")
    top = torch.topk(score, k, -1)
    return top.indices.int().contiguous(), torch.softmax(top.values, -1).contiguous()


@pytest.mark.parametrize("E,k,d,F", [(8, 1, 64, 64), (16, 4, 256, 192), (32, 8, 192, 320), (128, 4, 320, 128)])
@pytest.mark.parametrize("rows", [1, 5, 16, 63, 64, 65, 300, 1500])
def test_experts(E, k, d, F, rows):
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5, 1.0)
    y = ffn(lay, ex, m, ms, h, idx, w)
    assert torch.equal(y, by_products(E, d, F, ex, m, ms, h, idx, w))
    if rows <= 65:
        ref = I8.experts(m.cpu().numpy(), f64(ms), f64(h), idx.cpu().numpy(), f64(w), ex.gate_up.cpu().numpy(), f64(ex.gate_up_scale), ex.down.cpu().numpy(),
                         f64(ex.down_scale), lambda x: f64(torch.tensor(x).bfloat16()))
        # a row: its storage rounding, its experts' (2^-8 each), and codes that a rounding of silu(gate) * up moved by one, few and each
        # 1 / 127 of the largest
        err = np.linalg.norm(f64(y) - ref, axis=-1) / np.linalg.norm(ref, axis=-1)
        assert err.max() < 2 * 2.0 ** -8 + 2.0 ** -9, err.max()


def ffn_in_tiles(lay, mtile, ex, m, ms, h, idx, w):
    lay.ws = torch.empty(lay.moe_ffn_i8_workspace_bytes(m.shape[0]), dtype=torch.uint8, device="cuda")
    y, p = torch.empty_like(h), lambda t: C.c_void_p(t.data_ptr())
    e = B.ExpertsI8Struct(*(t.data_ptr() for t in (ex.gate_up, ex.gate_up_scale, ex.down, ex.down_scale)))
    lay.check(lay.L.compact_test_moe_ffn_i8(lay.ctx, C.c_int32(mtile), C.byref(e), p(m), p(ms), p(h), p(idx), p(w), C.c_int64(m.shape[0]), p(y), p(lay.ws),
                                            C.c_size_t(lay.ws.numel()), C.c_void_p(torch.cuda.current_stream().cuda_stream)))
    return y


@pytest.mark.parametrize("E,k,d,F", [(8, 2, 64, 64), (16, 4, 320, 192), (8, 3, 448, 640)])
@pytest.mark.parametrize("rows", [5, 40, 257, 900])
def test_experts_have_the_same_bits_at_every_row_tile_height(E, k, d, F, rows):
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5, 1.0)
    want = ffn(lay, ex, m, ms, h, idx, w)
    for mtile in (16, 64, 128, 256):
        assert torch.equal(ffn_in_tiles(lay, mtile, ex, m, ms, h, idx, w), want), mtile


@pytest.mark.parametrize("rows", [3, 16, 200])
def test_experts_with_indices_that_choose_none_or_one_twice(rows):
    E, k, d, F = 16, 4, 128, 64
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5)
    idx[0] = torch.tensor([-1, E, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)     # a row without an expert
    idx[1, 2], idx[2, 1] = -5, idx[2, 0]                                          # and one twice
    y = ffn(lay, ex, m, ms, h, idx, w)
    assert torch.equal(y[0], h[0]) and torch.equal(y, by_products(E, d, F, ex, m, ms, h, idx, w))
    idx[:] = -1
    assert torch.equal(ffn(lay, ex, m, ms, h, idx, w), h)
    idx[:] = 7                                                                    # all rows to one expert, four times
    assert torch.equal(ffn(lay, ex, m, ms, h, idx, w), by_products(E, d, F, ex, m, ms, h, idx, w))


def test_experts_in_place_and_a_broken_row():
    E, k, d, F = 16, 2, 128, 64
    for rows in (6, 150):
        lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
        m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
        idx, w = routed(rows, E, k, 5)
        ms[3] = math.nan
        y = ffn(lay, ex, m, ms, h, idx, w)
        assert y.isnan().any(-1).tolist() == [i == 3 for i in range(rows)] and bool(y[3].isnan().all())
        lay.compact_moe_ffn_i8(ex, m, ms, h, idx, w, h)
        assert torch.equal(h.view(torch.int16), y.view(torch.int16))


# ---- as a program runs them ------------------------------------------------------------------------------------------------------

class Chain:
    """The feed-forward half of a routed layer: norm and codes, routing, experts."""

    def __init__(self, rows, ws=None):
        self.lay, d = layer(d=256, F=192, E=16, k=4), 256
        self.ex, self.rule = experts(16, d, 192, 11), B.RouteRule("sigmoid", 4, 2, 2, factor=2.0)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.x, self.b, self.g, self.gate = rows_of(rows, d, "bf16", 1), rows_of(rows, d, "bf16", 3), torch.ones(d, **bf), torch.full((d,), 0.5, **bf)
        self.wr, self.bias = (0.1 * torch.randn((16, d), generator=gen(8), device="cuda")).bfloat16(), 0.1 * torch.randn(16, generator=gen(9), device="cuda")
        self.h, self.n, self.y = (torch.empty((rows, d), **bf) for _ in range(3))
        self.q, self.s = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        self.logits, self.w, self.idx = torch.empty((rows, 16), device="cuda"), torch.empty((rows, 4), device="cuda"), torch.empty((rows, 4), dtype=torch.int32, device="cuda")
        self.lay.ws = torch.empty(self.lay.moe_ffn_i8_workspace_bytes(rows), dtype=torch.uint8, device="cuda") if ws is None else ws

    def run(self):
        lay = self.lay
        lay.compact_block_norm(self.x, b=self.b, g_post=self.g, gate=self.gate, alpha=0.7, h=self.h, g_pre=self.g, n=self.n, q=self.q, q_scale=self.s)
        lay.compact_route(self.rule, self.logits, self.bias, self.idx, self.w, m=self.n, w_router=self.wr)
        lay.compact_moe_ffn_i8(self.ex, self.q, self.s, self.h, self.idx, self.w, self.y)
        return self.y


@pytest.mark.parametrize("rows", [7, 16, 333])
def test_a_captured_chain_replays_with_the_inputs_of_the_moment(rows):
    c = Chain(rows)
    want = c.run().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for turn in range(4):
        c.x.copy_(rows_of(rows, 256, "bf16", 20 + turn) if turn else rows_of(rows, 256, "bf16", 1))
        c.y.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        got = c.y.clone()
        assert torch.equal(got, c.run()), turn
        if turn == 0:
            assert torch.equal(got, want)
    # two graphs that share a workspace, one after the other
    d = Chain(rows, ws=c.lay.ws)
    d.x.copy_(rows_of(rows, 256, "bf16", 50))
    other = d.run().clone()
    torch.cuda.synchronize()
    g2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g2):
        d.run()
    for _ in range(3):
        d.y.zero_(), c.y.zero_()
        g2.replay(), graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d.y, other) and torch.equal(c.y, got)


def test_calls_on_side_streams_have_the_same_bits():
    a, b = Chain(100), Chain(100)
    want = a.run().clone()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for s, c in ((s1, a), (s2, b)):
            with torch.cuda.stream(s):
                c.y.zero_()
                c.run()
        torch.cuda.synchronize()
        assert torch.equal(a.y, want) and torch.equal(b.y, want)


# ---- offsets beyond 32 bits ------------------------------------------------------------------------------------------------------

def test_rows_of_more_than_4_gi_elements():
    n, d, k = 600_000, 8192, 5
    lay = layer(d=d)
    x = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    some = rows_of(k, d, "bf16", 1)
    x[:k], x[-k:] = some, some
    q, s = torch.full((n, d), 3, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    lay.compact_quant_i8(x, q, s)
    want, ws = quantised(lay, some)
    for at in (slice(0, k), slice(n - k, n)):
        assert torch.equal(q[at], want) and torch.equal(s[at], ws)
    assert int(q[k:-k:9973].abs().max()) == 0 and not s[k:-k].any()
    g, h = torch.ones(d, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    lay.compact_block_norm(x, b=x, h=h, g_pre=g, q=q, q_scale=s)
    h2, q2, s2 = torch.empty_like(some), torch.empty_like(want), torch.empty_like(ws)
    lay.compact_block_norm(some, b=some, h=h2, g_pre=g, q=q2, q_scale=s2)
    for at in (slice(0, k), slice(n - k, n)):
        assert torch.equal(q[at], q2) and torch.equal(s[at], s2) and torch.equal(h[at], h2)


@pytest.mark.parametrize("M,N,K", [(3, 40_000, 131_056), (300, 40_000, 131_056), (40_000, 24, 131_056), (70_000, 40_000, 32)])
def test_products_of_more_than_4_gi_elements(M, N, K):
    lay = layer()
    a, b = codes(M, K, 1), codes(N, K, 2)
    sa, sb = scales(M, 3), scales(N, 4) * 1e-6
    c = product(lay, a, sa, b, sb)
    rows, cols = sorted({0, M // 2, M - 2, M - 1}), sorted({0, 7, N // 2 + 1, N - 1})
    check_product(c[rows][:, cols], a[rows], sa[rows], b[cols], sb[cols], None, 0, "bf16")


def test_experts_of_more_than_4_gi_hidden_elements():
    E, k, d, F, rows = 8, 8, 64, 2944, 200_000
    lay, ex = layer(d=d, F=F, E=E, k=k), experts(E, d, F, 11)
    m, ms, h = codes(rows, d, 1), scales(rows, 2) / 70, rows_of(rows, d, "bf16", 3)
    idx, w = routed(rows, E, k, 5)
    y = ffn(lay, ex, m, ms, h, idx, w)
    for at in (slice(0, 40), slice(rows - 40, rows)):
        assert torch.equal(y[at], by_products(E, d, F, ex, m[at].contiguous(), ms[at].contiguous(), h[at].contiguous(), idx[at].contiguous(), w[at].contiguous()))


def test_routing_of_many_rows():
    lay, rows = layer(E=256, k=8), 9_000_000      # 2.3 gi logits
    x = torch.randn((1000, 256), generator=gen(1), device="cuda").repeat(rows // 1000, 1)
    idx, w = torch.empty((rows, 8), dtype=torch.int32, device="cuda"), torch.empty((rows, 8), device="cuda")
    for rule in (dict(score="sigmoid", n_groups=8, topk_groups=4, group_top=2), dict(score="softmax")):
        lay.compact_route(B.RouteRule(**rule), x, None, idx, w)
        i2, w2 = torch.empty((1000, 8), dtype=torch.int32, device="cuda"), torch.empty((1000, 8), device="cuda")
        lay.compact_route(B.RouteRule(**rule), x[:1000].contiguous(), None, i2, w2)
        assert torch.equal(idx.view(-1, 1000, 8), i2.expand(rows // 1000, -1, -1)) and torch.equal(w.view(-1, 1000, 8), w2.expand(rows // 1000, -1, -1))
