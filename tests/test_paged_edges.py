"""Paged cache in 8 bits, on the host: its definition at the top of the range, and what its calls refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged8 as P8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS, LayerConfig
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


class Calls:
    """Stands in for the library: counts the calls that reach it."""

    def __init__(self):
        self.n = 0

    def __getattr__(self, name):
        def call(*args):
            self.n += 1
            return 0
        return call


@pytest.fixture
def on_the_host(monkeypatch):
    """A layer whose calls end before the library, and what they take, on the CPU (whose device number is -1)."""
    lc = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=256, dtype="bf16")
    lay = B.Layer(lc, None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    real, lay.L = lay.L, Calls()
    yield lay, B.PagedKV.allocate(lc, 3, 4, 12, 16, "cpu")
    lay.L = real


def test_calls_refuse_arrays_that_are_not_on_the_current_gpu(on_the_host, monkeypatch):
    lay, kv = on_the_host
    lay.ws, st, bf = torch.zeros(1 << 20, dtype=torch.uint8), B.PagedStep(lay.layer, 3, 5, "cpu", n_pages=12), torch.bfloat16
    calls = (lambda: lay.compact_paged_plan(kv, st), lambda: lay.compact_rope_paged_write(torch.zeros((5, 768), dtype=bf), kv, st.slot, st.rot, torch.zeros((5, 512), dtype=bf)),
             lambda: lay.compact_attn_paged(torch.zeros((5, 512), dtype=bf), kv, st.cu, st.kv_len, 2, 64, torch.zeros((5, 512), dtype=bf)))
    for call in calls:
        call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in calls:
        assert refused(call)
    assert lay.L.n == 3


def refused(call):
    with pytest.raises(B.CompactError) as e:
        call()
    return e.value.code == 1


WRONG = [lambda t: t.float() if t.dtype is not torch.float32 else t.double(),           # another type
         lambda t: t.reshape(-1)[:-1],                                                  # one element short
         lambda t: t.reshape(-1).repeat_interleave(2)[::2].reshape(t.shape)]            # elements apart


def test_write_refuses_arrays_that_do_not_fit(on_the_host):
    lay, kv = on_the_host
    bf = torch.bfloat16
    good = dict(qkv=torch.zeros((5, 12 * 64), dtype=bf), slot=torch.zeros(5, dtype=torch.int64), rot=torch.zeros((5, 32, 2)), q=torch.zeros((5, 512), dtype=bf))

    def write(kv=kv, **over):
        a = dict(good, **over)
        lay.compact_rope_paged_write(a["qkv"], kv, a["slot"], a["rot"], a["q"])
    write()
    write(slot=torch.zeros(9, dtype=torch.int64), rot=torch.zeros((9, 32, 2)), q=torch.zeros((9, 512), dtype=bf))   # more rows are no harm
    write(qkv=torch.zeros((0, 12 * 64), dtype=bf))
    assert lay.L.n == 3
    for name in good:
        for wrong in WRONG:
            assert refused(lambda: write(**{name: wrong(good[name])})), name
    assert refused(lambda: write(slot=good["slot"].int()))
    assert refused(lambda: write(qkv=good["qkv"][:, :-64].contiguous()))
    other = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=4, head_dim=64, ffn_dim=256, dtype="bf16")
    assert refused(lambda: write(kv=B.PagedKV.allocate(other, 3, 4, 12, 16, "cpu")))
    assert lay.L.n == 3


def test_attention_refuses_arrays_that_do_not_fit(on_the_host):
    lay, kv = on_the_host
    bf = torch.bfloat16
    lay.ws = torch.zeros(1 << 20, dtype=torch.uint8)
    good = dict(q=torch.zeros((5, 512), dtype=bf), cu=torch.zeros(4, dtype=torch.int32), kv_len=torch.zeros(3, dtype=torch.int32), o=torch.zeros((5, 512), dtype=bf))

    def attn(kv=kv, **over):
        a = dict(good, **over)
        lay.compact_attn_paged(a["q"], kv, a["cu"], a["kv_len"], 2, 64, a["o"])
    attn()
    attn(q=torch.zeros((5, 768), dtype=bf)[:, :512])       # rows may be apart
    attn(cu=torch.zeros(9, dtype=torch.int32), o=torch.zeros((9, 512), dtype=bf))
    assert lay.L.n == 3
    for name in ("cu", "kv_len", "o"):
        for wrong in WRONG:
            assert refused(lambda: attn(**{name: wrong(good[name])})), name
    assert refused(lambda: attn(q=good["q"].reshape(-1)))
    assert refused(lambda: attn(q=good["q"].float())) and refused(lambda: attn(q=good["q"][:, :-8])) and refused(lambda: attn(q=torch.zeros((512, 5), dtype=bf).T))
    other = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=1, head_dim=128, ffn_dim=256, dtype="bf16")
    assert refused(lambda: attn(kv=B.PagedKV.allocate(other, 3, 4, 12, 16, "cpu")))
    assert lay.L.n == 3


def test_plan_refuses_arrays_that_do_not_fit(on_the_host):
    lay, kv = on_the_host

    def step(**over):
        st = B.PagedStep(lay.layer, 3, 40, "cpu", n_pages=12)
        for name, value in over.items():
            setattr(st, name, value)
        lay.compact_paged_plan(kv, st)
    step()
    assert lay.L.n == 1
    st = B.PagedStep(lay.layer, 3, 40, "cpu", n_pages=12)
    for name in ("n_new", "len", "n_free", "free", "n_free_out", "n_refused", "len_out", "kv_len", "cu", "slot", "rot"):
        for wrong in WRONG:
            t = wrong(getattr(st, name))
            if t.numel() > 1 or t.is_contiguous() and (t.dtype is not getattr(st, name).dtype or t.numel() == 0):   # (one element is never apart)
                assert refused(lambda: step(**{name: t})), name
    assert refused(lambda: lay.compact_paged_plan(kv, B.PagedStep(lay.layer, 2, 40, "cpu", n_pages=12)))
    assert refused(lambda: lay.compact_paged_plan(kv, B.PagedStep(lay.layer, 3, 40, "cpu", n_pages=11)))
    wide = LayerConfig(d_model=512, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn_dim=256, dtype="bf16")
    assert refused(lambda: lay.compact_paged_plan(kv, B.PagedStep(wide, 3, 40, "cpu", n_pages=12)))     # its rows of `rot` are not the layer's
    assert lay.L.n == 1


def test_a_cache_refuses_pages_of_other_shapes():
    lc = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=256, dtype="bf16")
    kv = B.PagedKV.allocate(lc, 3, 4, 12, 16, "cpu")
    good = dict(k=kv.k, v=kv.v, k_scale=kv.k_scale, v_scale=kv.v_scale, table=kv.table)
    B.PagedKV(lc, **good)
    for name in ("k", "v", "k_scale", "v_scale"):
        for bad in (good[name][:-1], good[name].float(), good[name].transpose(0, 1).contiguous().transpose(0, 1)):
            assert refused(lambda: B.PagedKV(lc, **dict(good, **{name: bad}))), name
    for bad in (kv.table.long(), kv.table.t().contiguous().t()):
        assert refused(lambda: B.PagedKV(lc, **dict(good, table=bad)))


def test_a_cache_whose_arrays_are_replaced_uses_the_new_ones(on_the_host):
    lay, kv = on_the_host
    st, seen = B.PagedStep(lay.layer, 3, 5, "cpu", n_pages=20), []

    def plan():
        lay.L.compact_paged_plan = lambda ctx, ref, step, stream: seen.append(ref._obj) or 0
        lay.compact_paged_plan(kv, st)
        return seen[-1]
    assert (plan().d_table, plan().d_k, plan().n_pages) == (kv.table.data_ptr(), kv.k.data_ptr(), 12)
    kv.table = torch.full((3, 6), -1, dtype=torch.int32)
    assert (plan().d_table, plan().max_pages, kv.max_pages) == (kv.table.data_ptr(), 6, 6)
    big = B.PagedKV.allocate(lay.layer, 3, 6, 20, 16, "cpu")       # a larger pool, array by array
    kv.k, kv.v, kv.k_scale, kv.v_scale = big.k, big.v, big.k_scale, big.v_scale
    assert refused(plan)                                             # the number of pages is still the old one
    kv.n_pages = 20
    c = plan()
    assert (c.d_k, c.d_v, c.d_k_scale, c.d_v_scale, c.n_pages) == (big.k.data_ptr(), big.v.data_ptr(), big.k_scale.data_ptr(), big.v_scale.data_ptr(), 20)
    kv.table = torch.full((2, 6), -1, dtype=torch.int32)
    assert refused(plan)                                             # the step has three requests


def pieces(n, kv, G):
    """Into how many pieces a request's keys are cut (n rows of G query heads each per KV head)."""
    if n <= 32 and n * G <= 32:
        return max(-(-kv // 256), 1)
    tiles = -(-n * G // 128)
    return max(kv // 512 // tiles, min(kv // 2048, 64 // tiles), 1)


def wide(G):
    return B.Layer(LayerConfig(d_model=4096, n_q_heads=8 * G, n_kv_heads=8, head_dim=128, ffn_dim=4096, dtype="bf16"), None)


@pytest.mark.parametrize("n_requests,max_kv,mib", [(24, 8192, 340), (512, 8192, 1050), (512, 32768, 4200), (1, 8192, 40), (4096, 2048, 270)])
def test_workspace_goes_by_the_rows_of_a_call(n_requests, max_kv, mib):
    """2048 rows a step, all of which one request may bring: no slot has room for all of them by itself."""
    lay = wide(4)
    assert lay.paged_workspace_bytes(n_requests, 2048, 2048, max_kv) <= mib << 20
    # never more than a record for every row, query head and 256 keys, nor than the requests' own by themselves
    base = lay.paged_workspace_bytes(1, 1, 1, 1)
    assert lay.paged_workspace_bytes(n_requests, 2048, 2048, max_kv) - base <= 2048 * -(-max_kv // 256) * 32 * 130 * 4
    assert lay.paged_workspace_bytes(n_requests, 2048, 2048, max_kv) - base <= n_requests * (lay.paged_workspace_bytes(1, 1 << 20, 2048, max_kv) - base)


@pytest.mark.parametrize("G", [1, 3, 4, 16])
def test_workspace_holds_every_batch_and_grows_with_each_bound(G):
    lay, rng = wide(G), np.random.default_rng(G)
    base = lay.paged_workspace_bytes(1, 1, 1, 1)
    for _ in range(500):
        N, most, max_kv = int(rng.integers(1, 40)), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 17))
        few = min(most, 32 // G)
        n = [int(rng.choice([1, few, min(few + 1, most), most, rng.integers(0, most + 1)])) for _ in range(N)]
        kv = [int(rng.choice([max_kv, rng.integers(0, max_kv + 1)])) for _ in range(N)]
        rows, need = max(sum(n), 1), sum(a * pieces(a, b, G) for a, b in zip(n, kv) if pieces(a, b, G) > 1)
        have = lay.paged_workspace_bytes(N, rows, most, max_kv)
        assert have - base >= need * 8 * G * 130 * 4, (n, kv)
        for more in ((N + 1, rows, most, max_kv), (N, rows + 9, most, max_kv), (N, rows, most + 5, max_kv), (N, rows, most, max_kv + 300)):
            assert lay.paged_workspace_bytes(*more) >= have, (more, n)


def test_a_step_that_advances_swaps_its_arrays():
    lc = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=256, dtype="bf16")
    st = B.PagedStep(lc, 3, 5, "cpu", n_pages=12)
    st.advance()                              # before its first call as well
    for _ in range(3):
        before = st.struct() and (st.len, st.n_free)
        st.advance()
        assert st.len_out is before[0] and st.n_free_out is before[1]
        names = [n for n, _ in B.PagedStepStruct._fields_[:-1]]
        assert [getattr(st.struct(), n) for n in names] == [getattr(st, n[2:]).data_ptr() for n in names]
    st.len = torch.zeros(4, dtype=torch.int32)
    assert refused(st.struct)
