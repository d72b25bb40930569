"""Paged cache in 8 bits, on the host: pins of its plain definition, and what the calls refuse before touching the device."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged8 as P8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import WORKLOADS, LayerConfig


def test_e4m3_values_are_those_of_the_format():
    v = P8.VALUES
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and np.isfinite(np.delete(v, [0x7F, 0xFF])).all()
    assert (v[0x00], v[0x01], v[0x08], v[0x38], v[0x7E], v[0xFE]) == (0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -448.0)
    mine = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mine, v, equal_nan=True)


def test_rounding_to_e4m3():
    finite = [c for c in range(256) if c & 127 != 127]
    assert P8.to_e4m3(P8.VALUES[finite]).tolist() == finite
    # halfway cases go to the even code, the values around them to the nearest
    for c in range(126):
        mid = (P8.VALUES[c] + P8.VALUES[c + 1]) / 2
        assert P8.to_e4m3(mid) == c + (c & 1) and P8.to_e4m3(-mid) == 128 + c + (c & 1)
        assert P8.to_e4m3(mid * (1 - 1e-9)) == c and P8.to_e4m3(mid * (1 + 1e-9)) == c + 1
    assert P8.to_e4m3(np.nan) == 127


@pytest.mark.parametrize("e", [-100, -9, 0, 3, 90])
def test_scale_is_the_least_power_of_two(e):
    assert P8.scale_byte(448.0 * 2.0 ** e) == e + 127
    assert P8.scale_byte(448.0 * 2.0 ** e * (1 + 1e-12)) == e + 128
    assert P8.scale_byte(224.0 * 2.0 ** e * (1 + 1e-12)) == e + 127
    assert P8.scale_byte(0.0) == 1


def test_plan_by_hand():
    # pages of 16; request 0 decodes into a new page, 1 rests, 2 has finished (its two pages go on the stack), 3 needs four
    # pages and is refused (three are left), 4 goes on inside its page, 5 takes one of the three
    table = [[4, -1, -1, -1], [5, -1, -1, -1], [6, 7, -1, -1], [-1] * 4, [8, -1, -1, -1], [-1] * 4]
    out = P8.plan([1, 0, -1, 64, 3, 2], [16, 5, 20, 0, 4, 0], [0, 1, 9, 9], 2, table, 16, 70 + 3)
    assert out["n_refused"] == 2      # 3, and 5: the pages wanted up to and including it are more than there are
    assert out["cu"] == [0, 1, 1, 1, 65, 68, 70] and out["len"] == [17, 5, 0, 0, 7, 0] and out["kv_len"] == [17, 0, 0, 0, 7, 0]
    assert out["table"][0] == [4, 7, -1, -1] and out["table"][4] == table[4] and out["table"][5] == table[5]
    assert out["slot"][:2] == [7 * 16, -1] and out["slot"][65:70] == [8 * 16 + 4, 8 * 16 + 5, 8 * 16 + 6, -1, -1]
    assert out["n_free"] == 3 and out["free"][:3] == [0, 1, 6]


def test_pages_by_hand():
    p = P8.Pages(2, 16, 1, 2)
    row = lambda *x: np.array(x, dtype=np.float64).reshape(-1, 1, 2)   # noqa: E731
    p.write([16], row(448.0, 2.0 ** -9), row(1.0, -1.0))
    assert p.scale["k"][1, 0] == 127 and p.scale["v"][1, 0] == 127 - 8
    p.write([17], row(449.0, 1.0), row(0.5, np.inf))      # K's scale doubles; 2^-9 is half the smallest code of the new scale
    assert p.scale["k"][1, 0] == 128 and p.scale["v"][1, 0] == 127 - 8
    assert p.rows("k", [1], 1).ravel().tolist() == [448.0, 0.0]
    assert np.isnan(p.rows("k", [1], 2)[1]).all() and p.rows("v", [1], 2)[1].ravel().tolist() == [0.5, 0.0]


def _kv(**over):
    kw = dict(d_k=0x10000, d_v=0x20000, d_k_scale=0x30000, d_v_scale=0x40000, d_table=0x50000, n_pages=64, page_rows=64, max_pages=16, n_requests=4)
    kw.update(over)
    return B.PagedKVStruct(*[kw[n] for n, _ in B.PagedKVStruct._fields_])


def _step(**over):
    names = [n for n, _ in B.PagedStepStruct._fields_]
    kw = {n: 0x1000 * (i + 1) for i, n in enumerate(names)}
    kw["max_rows"] = 64
    kw.update(over)
    return B.PagedStepStruct(*[kw[n] for n in names])


BAD_CACHES = [(dict(d_table=None), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(n_requests=0), 1), (dict(n_requests=4097), 2),
              (dict(page_rows=8), 2), (dict(page_rows=48), 2), (dict(page_rows=256), 2), (dict(page_rows=0), 2),
              (dict(max_pages=1 << 25), 2)]


def test_paged_calls_reject_bad_arguments_without_a_device():
    lay = B.Layer(WORKLOADS["dense_8x4096"].layer, None)
    L, ctx, p = lay.L, lay.ctx, C.c_void_p(0x60000)

    def plan(kv=_kv(), st=_step()):
        return L.compact_paged_plan(ctx, C.byref(kv) if kv is not None else None, C.byref(st) if st is not None else None, None)

    def write(kv=_kv(), n=8, qkv=p, slot=p, rot=p, q=p):
        return L.compact_rope_paged_write(ctx, n, qkv, C.byref(kv) if kv is not None else None, slot, rot, q, None)

    def attn(kv=_kv(), n=8, cu=p, kvl=p, new=2, most=1024, q=p, stride=4096, o=p, ws=p, wsn=1 << 40):
        return L.compact_attn_paged(ctx, C.byref(kv) if kv is not None else None, n, cu, kvl, new, most, q, stride, o, ws, wsn, None)

    for call in (plan, write, attn):
        assert call(kv=None) == 1
        for kw, code in BAD_CACHES:
            assert call(kv=_kv(**kw)) == code, kw
            assert L.compact_last_error(ctx) != b""
    for call in (write, attn):      # a plan needs no pages
        for kw in (dict(d_k=None), dict(d_v=None), dict(d_k_scale=None), dict(d_v_scale=None), dict(d_k=0x10008), dict(d_v=0x20001)):
            assert call(kv=_kv(**kw)) == 1, kw
    assert plan(st=None) == 1
    for n, _ in B.PagedStepStruct._fields_[:-1]:
        assert plan(st=_step(**{n: None})) == 1, n
    assert plan(st=_step(max_rows=0)) == 1
    assert plan(st=_step(max_rows=(1 << 30) + 1)) == 2
    assert plan(st=_step(d_len_out=_step().d_len)) == 1           # lengths in and out are two arrays
    assert plan(st=_step(d_n_free_out=_step().d_n_free)) == 1
    assert plan(st=_step(d_rot=0xB004)) == 1
    assert write(n=-1) == 1
    for kw in (dict(qkv=None), dict(slot=None), dict(rot=None), dict(q=None), dict(qkv=C.c_void_p(0x60008)), dict(q=C.c_void_p(0x60002)),
               dict(slot=C.c_void_p(0x60004)), dict(rot=C.c_void_p(0x60004))):
        assert write(**kw) == 1, kw
    for kw, code in ((dict(n=-1), 1), (dict(n=(1 << 26) + 1), 2), (dict(cu=None), 1), (dict(kvl=None), 1), (dict(q=None), 1), (dict(o=None), 1),
                     (dict(new=0), 1), (dict(most=0), 1), (dict(stride=4088), 1), (dict(stride=4100), 1), (dict(q=C.c_void_p(0x60008)), 1),
                     (dict(ws=None), 4), (dict(wsn=1024), 4), (dict(ws=C.c_void_p(0x60004)), 4)):
        assert attn(**kw) == code, kw
    # nothing to do: nothing is launched
    assert write(n=0) == 0 and attn(n=0) == 0


def test_paged_workspace_grows_with_what_is_split():
    lay = B.Layer(LayerConfig(d_model=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, ffn_dim=4096, dtype="bf16"), None)
    base = lay.paged_workspace_bytes(8, 8, 1, 256)
    assert lay.paged_workspace_bytes(64, 64, 1, 256) == base                      # nobody's keys are split
    rec = lay.paged_workspace_bytes(8, 8, 1, 1024) - base
    assert rec >= 8 * 4 * 32 * (128 + 2) * 4                                       # a record per 256 keys and query head
    assert lay.paged_workspace_bytes(16, 16, 1, 1024) - base == 2 * rec
    assert lay.paged_workspace_bytes(8, 4096, 512, 1023) >= base
    assert lay.paged_workspace_bytes(8, 8, 512, 32768) == lay.paged_workspace_bytes(8, 8, 8, 32768)   # no more rows than there are
    for bad in ((0, 8, 1, 256), (8, -1, 1, 256), (8, 8, 0, 256), (8, 8, 1, 0)):
        with pytest.raises(B.CompactError) as e:
            lay.paged_workspace_bytes(*bad)
        assert e.value.code == 1
