"""8-bit integer weights on the host: the definition, and what the calls refuse."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import int8 as I8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS, LayerConfig
from tests.test_paged_edges import Calls, refused

ROUTED = LayerConfig(d_model=128, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=64, n_experts=16, top_k=4, dtype="bf16")


def half_even(f):
    n, rest = divmod(f, 1)
    return int(n) + (1 if rest > Fraction(1, 2) or rest == Fraction(1, 2) and n % 2 else 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_are_the_nearest_of_the_exact_quotient(dtype):
    x = torch.randn((40, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    x[3, 5], x[4, :2] = x[3].abs().max() / 2, torch.tensor([3.0, -1.5])     # ties: half of the largest
    x[5] = 0
    x[6, 0], x[7, 1], x[8, 2] = float("inf"), float("nan"), -float("inf")
    q, scale = I8.row_codes(x.double().numpy())
    for i in range(40):
        row = x[i].double().tolist()
        if i in (6, 7, 8):
            assert np.isnan(scale[i]) and not q[i].any()
            continue
        amax = max(abs(v) for v in row)
        assert scale[i] == np.float32(amax) / np.float32(127)
        assert q[i].tolist() == [half_even(127 * Fraction(v) / Fraction(amax)) if amax else 0 for v in row]
    assert q[3, 5] in (64, -64) and abs(q).max() == 127


def test_products_and_norms_of_hand_worked_rows():
    a, b = np.array([[127, -128, 0], [1, 2, 3]]), np.array([[127, -128, 1], [-1, 0, 5]])
    assert I8.product(a, [0.5, 1.0], b, [1.0, 0.25]).tolist() == [[0.5 * (127 * 127 + 128 * 128), -127 * 0.125], [127 - 256 + 3, 3.5]]
    x, br = np.array([[1.0, 2.0]]), np.array([[3.0, 4.0]])
    assert np.allclose(I8.residual(x, br, np.array([1.0, 2.0]), np.array([0.5, 1.0]), 2.0, 0.0), [[1 + 3 / 12.5 ** 0.5, 2 + 16 / 12.5 ** 0.5]])
    assert I8.residual(x, br, None, None, 0.5, 0.0).tolist() == [[2.5, 4.0]]


def test_routing_by_hand():
    l = np.log(np.array([[1.0, 3.0, 2.0, 3.0, 1.0, 6.0]]))
    idx, w, _ = I8.route(l, None, 3, "softmax", renorm=False)
    assert idx.tolist() == [[5, 1, 3]] and np.allclose(w, [[6 / 16, 3 / 16, 3 / 16]])
    idx, w, _ = I8.route(l, None, 2, "softmax", renorm=True, factor=2.5)
    assert idx.tolist() == [[5, 1]] and np.allclose(w, [[2.5 * 6 / 9, 2.5 * 3 / 9]])
    # groups {0,1} {2,3} {4,5}: the best two have 5/16 and 7/16
    idx, _, _ = I8.route(l, None, 3, "softmax", 3, 2, 2)
    assert idx.tolist() == [[5, 3, 2]]
    # a bias moves the choice, not the weight; a dead expert is the last choice and weighs nothing
    idx, w, _ = I8.route(l, np.array([9, 0, 0, 0, 0, 0.0]), 1, "softmax", renorm=False)
    assert idx.tolist() == [[0]] and np.allclose(w, [[1 / 16]])
    idx, w, _ = I8.route(np.array([[-np.inf, 0.0, np.nan, 1.0]]), np.array([9, 0, 9, 0.0]), 3, "sigmoid")
    assert idx.tolist() == [[3, 1, 0]] and w[0, 2] == 0 and np.isclose(w.sum(), 1)
    idx, w, _ = I8.route(np.full((1, 4), -np.inf), None, 2, "softmax")
    assert idx.tolist() == [[0, 1]] and w.tolist() == [[0, 0]]


# ---- refusals ----------------------------------------------------------------------------------------------------------------

P = 0x1000   # an address that no kernel ever sees


def code(lay, name, *args):
    return getattr(lay.L, name)(lay.ctx, *args)


def test_calls_refuse_what_the_kernels_cannot_take():
    lay = B.Layer(WORKLOADS["dense_8x4096"].layer, None)
    n = C.c_size_t()
    for args in ((P, 64, -1, 64, P, P), (P, 64, 1, 0, P, P), (P, 63, 2, 64, P, P), (None, 64, 1, 64, P, P), (P, 64, 1, 64, None, P), (P, 64, 1, 64, P, None),
                 (P + 1, 64, 1, 64, P, P)):
        assert code(lay, "compact_quant_i8", *args, None) == 1, args
    assert code(lay, "compact_quant_i8", P, 64, 1 << 31, 64, P, P, None) == 2
    good = [P, P, P, P, None, P, 4, 64, 64, 0]
    for at, v, rc in ((0, None, 1), (1, None, 1), (2, None, 1), (3, None, 1), (5, None, 1), (6, -1, 1), (7, 0, 1), (8, 0, 1), (9, 2, 1), (8, 72, 2), (8, 131072, 2),
                      (0, P + 8, 1), (2, P + 4, 1), (5, P + 8, 1), (4, P + 8, 1), (7, 1 << 30, 2)):
        args = list(good)
        args[at] = v
        assert code(lay, "compact_gemm_i8", *args, None, 0, None) == rc, (at, v)
    assert code(lay, "compact_gemm_i8", P, P, P, P, P, P, 4, 64, 64, 1, None, 0, None) == 1      # a residual behind SwiGLU
    assert code(lay, "compact_gemm_i8_workspace_bytes", 4, 64, 72, 0, C.byref(n)) == 2
    assert code(lay, "compact_gemm_i8_workspace_bytes", 4, 64, 64, 0, None) == 1
    good = [P, P, P, P, 0, 1.0, P, P, 2 * P, P, P, 4]
    for change in ({6: None, 8: None, 9: None, 10: None}, {9: None}, {10: None}, {7: None}, {1: None}, {1: None, 2: None, 3: None}, {0: None}, {4: 4}, {4: 4092}, {4: -4096},
                   {11: -1}, {0: P + 8}, {2: P + 8}, {9: P + 4}, {8: P}):
        args = [change.get(i, v) for i, v in enumerate(good)]
        assert code(lay, "compact_block_norm", *args, None) == 1, change
    assert code(lay, "compact_block_norm", *good[:-1], 1 << 31, None) == 2
    # nothing to do: nothing is looked at
    assert code(lay, "compact_quant_i8", None, 64, 0, 64, None, None, None) == 0
    assert code(lay, "compact_gemm_i8", None, None, None, None, None, None, 0, 64, 64, 0, None, 0, None) == 0
    assert code(lay, "compact_block_norm", None, None, P, P, 0, 1.0, None, P, None, None, None, 0, None) == 0
    assert code(lay, "compact_block_norm", None, None, P, P, 0, 1.0, None, P, None, None, P, 0, None) == 0   # arrays without rows have no address
    assert code(lay, "compact_block_norm", None, None, P, P, 0, 1.0, None, P, None, None, None, -1, None) == 1


def test_routing_refuses_rules_that_do_not_fit():
    lay = B.Layer(ROUTED, None)

    def route(lay=lay, m=None, w=None, rows=4, logits=P, **rule):
        r = dict(dict(score=0, n_groups=4, topk_groups=2, group_top=2, renorm=1, factor=1.0), **rule)
        return code(lay, "compact_route", C.byref(B.RouteRuleStruct(*r.values())), m, w, logits, None, rows, P, P, None)
    assert route(score=2) == 1 and route(score=-1) == 1 and route(group_top=0) == 1 and route(group_top=3) == 1
    assert route(n_groups=0) == 2 and route(n_groups=3) == 2 and route(topk_groups=0) == 2 and route(topk_groups=5) == 2
    assert route(n_groups=16, topk_groups=3) == 2      # fewer experts than top_k
    assert route(m=P) == 1 and route(w=P) == 1 and route(logits=None) == 1 and route(rows=-1) == 1 and route(rows=1 << 31) == 2
    assert route(m=P, w=P + 8) == 1 and route(m=P + 2, w=P) == 1 and route(m=P, w=P, logits=P + 4) == 1
    assert route(rows=0, logits=None) == 0 and route(rows=0, logits=None, w=P) == 0 and route(rows=0, n_groups=3) == 2
    assert code(lay, "compact_route", None, None, None, P, None, 4, P, P, None) == 1
    assert route(lay=B.Layer(WORKLOADS["dense_8x4096"].layer, None)) == 1
    assert refused(lambda: B.RouteRule(score="tanh"))
    for wrong in (dict(n_groups=2 ** 32 + 4), dict(n_groups=4, topk_groups=2 ** 32 + 2), dict(group_top=2 ** 32 + 1), dict(n_groups=1 - 2 ** 32)):
        assert refused(lambda: B.RouteRule(**wrong)), wrong


def test_experts_refuse_what_the_kernels_cannot_take():
    lay, n = B.Layer(ROUTED, None), C.c_size_t()

    def ffn(lay=lay, w=(P, P, P, P), rows=4, m=P, h=P, ws=P, size=1 << 30):
        return code(lay, "compact_moe_ffn_i8", C.byref(B.ExpertsI8Struct(*w)), m, P, h, P, P, rows, P, ws, size, None)
    for i in range(4):
        assert ffn(w=tuple(None if j == i else P for j in range(4))) == 1
    assert ffn(m=None) == 1 and ffn(m=P + 8) == 1 and ffn(h=P + 2) == 1 and ffn(rows=-1) == 1 and ffn(rows=(1 << 24) + 1) == 2
    need = lay.moe_ffn_i8_workspace_bytes(4)
    assert ffn(ws=None) == 4 and ffn(size=need - 1) == 4
    assert ffn(rows=0, m=None, ws=None, size=0) == 0
    assert ffn(lay=B.Layer(WORKLOADS["dense_8x4096"].layer, None)) == 1
    fp32 = B.Layer(LayerConfig(**dict(ROUTED.as_dict(), dtype="fp32")), None)
    assert ffn(lay=fp32) == 5 and code(fp32, "compact_moe_ffn_i8_workspace_bytes", 4, C.byref(n)) == 5


@pytest.fixture
def on_the_host(monkeypatch):
    lay = B.Layer(ROUTED, None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    real, lay.L = lay.L, Calls()
    yield lay
    lay.L = real


WRONG = [lambda t: t.float() if t.dtype is not torch.float32 else t.double(), lambda t: t.reshape(-1)[:-1],
         lambda t: t.reshape(-1).repeat_interleave(2)[::2].reshape(t.shape)]


def arrays():
    bf, i8 = torch.bfloat16, torch.int8
    z = torch.zeros
    return dict(
        quant=dict(x=z((5, 24), dtype=bf), q=z((5, 24), dtype=i8), scale=z(5)),
        gemm=dict(a=z((5, 32), dtype=i8), a_scale=z(5), b=z((12, 32), dtype=i8), b_scale=z(12), r=z((5, 12), dtype=bf), c=z((5, 12), dtype=bf)),
        norm=dict(x=z((5, 128), dtype=bf), b=z((5, 128), dtype=bf), g_post=z(128, dtype=bf), gate=z((5, 128), dtype=bf), h=z((5, 128), dtype=bf),
                  g_pre=z(128, dtype=bf), n=z((5, 128), dtype=bf), q=z((5, 128), dtype=i8), q_scale=z(5)),
        route=dict(logits=z((5, 16)), bias=z(16), idx=z((5, 4), dtype=torch.int32), weight=z((5, 4)), m=z((5, 128), dtype=bf), w_router=z((16, 128), dtype=bf)),
        moe=dict(gate_up=z((16, 128, 128), dtype=i8), gate_up_scale=z((16, 128)), down=z((16, 128, 64), dtype=i8), down_scale=z((16, 128)), m=z((5, 128), dtype=i8),
                 m_scale=z(5), h=z((5, 128), dtype=bf), idx=z((5, 4), dtype=torch.int32), weight=z((5, 4)), y=z((5, 128), dtype=bf)))


def call(lay, op, a):
    if op == "quant":
        lay.compact_quant_i8(a["x"], a["q"], a["scale"])
    elif op == "gemm":
        lay.compact_gemm_i8(a["a"], a["a_scale"], a["b"], a["b_scale"], a["r"], a["c"])
    elif op == "norm":
        lay.compact_block_norm(**a)
    elif op == "route":
        lay.compact_route(B.RouteRule(), a["logits"], a["bias"], a["idx"], a["weight"], a["m"], a["w_router"])
    else:
        lay.compact_moe_ffn_i8(B.ExpertsI8(a["gate_up"], a["gate_up_scale"], a["down"], a["down_scale"]), *(a[k] for k in ("m", "m_scale", "h", "idx", "weight", "y")))


# rows of quant's x and of a gate may be apart; elements may not
@pytest.mark.parametrize("op,name", [(op, name) for op, a in arrays().items() for name in a])
def test_arrays_that_do_not_fit_are_refused(on_the_host, op, name):
    lay, good = on_the_host, arrays()[op]
    lay.ws = torch.zeros(1 << 20, dtype=torch.uint8)
    call(lay, op, good)
    assert lay.L.n == 1
    for wrong in WRONG:
        assert refused(lambda: call(lay, op, dict(good, **{name: wrong(good[name])}))), name
    assert lay.L.n == 1


def test_arrays_that_may_be_refused_or_not(on_the_host, monkeypatch):
    lay, a = on_the_host, arrays()
    lay.compact_quant_i8(torch.zeros((5, 48), dtype=torch.bfloat16)[:, 8:32], a["quant"]["q"], a["quant"]["scale"])
    assert refused(lambda: lay.compact_quant_i8(torch.zeros((24, 5), dtype=torch.bfloat16).T, a["quant"]["q"], a["quant"]["scale"]))
    call(lay, "gemm", dict(a["gemm"], r=None))
    g = dict(a["gemm"], b=torch.zeros((24, 32), dtype=torch.int8), b_scale=torch.zeros(24), r=None)
    lay.compact_gemm_i8(*(g[k] for k in ("a", "a_scale", "b", "b_scale", "r", "c")), epilogue=1)
    assert refused(lambda: call(lay, "gemm", g))       # rows for SwiGLU without it
    assert refused(lambda: call(lay, "gemm", dict(a["gemm"], a=torch.zeros((5, 48), dtype=torch.int8))))
    call(lay, "norm", dict(a["norm"], gate=torch.zeros(128, dtype=torch.bfloat16)))
    call(lay, "norm", dict(a["norm"], gate=torch.zeros((5, 256), dtype=torch.bfloat16)[:, :128]))
    call(lay, "route", dict(a["route"], bias=None, m=None, w_router=None))
    assert lay.L.n == 6
    lay.ws = torch.zeros(16, dtype=torch.uint8, device="meta")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for op in a:
        assert refused(lambda: call(lay, op, a[op])), op
    assert lay.L.n == 6


def test_sizes_beyond_32_bits_are_refused(on_the_host):
    lay, n, bf, i8 = on_the_host, 2 ** 32 + 64, torch.bfloat16, torch.int8

    def z(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")
    lay.compact_gemm_i8(z(1, 16, dtype=i8), z(1), z(8, 16, dtype=i8), z(8), None, z(1, 8, dtype=bf))
    lay.compact_quant_i8(z(1, 64, dtype=bf), z(1, 64, dtype=i8), z(1))
    assert lay.L.n == 2
    assert refused(lambda: lay.compact_quant_i8(z(1, n, dtype=bf), z(1, n, dtype=i8), z(1)))
    assert refused(lambda: lay.compact_gemm_i8(z(1, n, dtype=i8), z(1), z(1, n, dtype=i8), z(1), None, z(1, 1, dtype=bf)))
    assert refused(lambda: lay.compact_gemm_i8(z(1, 16, dtype=i8), z(1), z(n, 16, dtype=i8), z(n), None, z(1, n, dtype=bf)))
    assert lay.L.n == 2
