"""Paged cache in 8 bits at the edges of what its calls accept: requests without cached rows beside pages that hold anything,
values at the top of the range, stacks of as many pages as there are numbers, arrays that are not on the GPU,
workspaces of exactly the size that is asked for."""
import pytest
import torch

from paper_2605_23296_amd import binding as B
from tests.test_gpu_paged import ATTN_LAYERS, DEV, IDS, check_attn, handle, ints, layer, queries, random_cache, run_attn, tdtype

pytestmark = pytest.mark.gpu


def with_nobodys_page_0(kv, ref, table):
    """The same cache behind one more page that no request owns, full of NaN codes and NaN scales."""
    def behind(x, fill):
        return torch.cat([torch.full_like(x[:1], fill), x])
    kv = B.PagedKV(kv.layer, behind(kv.k, 0x7F), behind(kv.v, 0x7F), behind(kv.k_scale, 255), behind(kv.v_scale, 255), kv.table + (kv.table >= 0).int())
    return kv


@pytest.mark.parametrize("lc", ATTN_LAYERS, ids=IDS)
@pytest.mark.parametrize("n_new,lens", [([1, 1, 1], [0, 300, 0]), ([4, 2, 1], [0, 40, 0]), ([1, 4, 1, 90, 2], [0, 0, 300, 100, 0])],
                         ids=["single_tokens", "a_few_rows", "beside_a_prompt"])
@pytest.mark.parametrize("entry", [-1, 0])
def test_requests_without_cached_rows_give_zeros(lc, n_new, lens, entry):
    """As the plan leaves a request that it refused: rows in the batch, no cached ones, and a table row that names nothing or a page
    of somebody else's, here one whose codes and scales are NaN."""
    kv, ref, table = random_cache(lc, lens, 32, 21)
    kv = with_nobodys_page_0(kv, ref, table)
    for i, L in enumerate(lens):
        if L == 0:
            kv.table[i].fill_(entry)
    q, lay = queries(lc, sum(n_new), 21), handle(lc)
    o = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, o, n_new, lens, ref, table)
    for rows, L in zip(torch.split(o, n_new), lens):
        assert L > 0 or (rows == 0).all()


@pytest.mark.parametrize("lc", [layer(8, 2, 128), layer(8, 2, 64), layer(4, 2, 64, "fp32"), layer(4, 2, 128, "fp32")], ids=IDS)
@pytest.mark.parametrize("T,n,at", [(290, 1, None), (290, 3, 288), (66, 4, 64), (200, 200, 96), (700, 130, 640)])
@pytest.mark.parametrize("name", ["k", "v"])
def test_the_largest_finite_values_leave_rows_that_do_not_see_them_alone(lc, T, n, at, name):
    """A cached row (the first one of a page) with the storage type's largest values in one KV head: what is read back is finite and within
    a code's rounding, and the rows before it have the bits that they have beside an ordinary row."""
    H, Hq, hd, P, dt = lc.n_kv_heads, lc.n_q_heads, lc.head_dim, 32, tdtype(lc)
    big, lay = torch.finfo(dt).max, handle(lc)
    g = torch.Generator().manual_seed(22)
    plain = torch.randn((T, Hq + 2 * H, hd), generator=g).to(dt)
    at = T - 1 if at is None else at
    large = plain.clone()
    if name == "k":      # (its rotation stays within the type: the other half is 0)
        large[at, Hq + 1] = 0.0
        large[at, Hq + 1, :2] = torch.tensor([big, -big])
    else:
        large[at, Hq + H + 1, :4] = torch.tensor([big, -big, big / 2, 248 * 2.0 ** 120])
    out = []
    for x in (plain, large):
        kv = B.PagedKV.allocate(lc, 1, -(-T // P), -(-T // P), P, DEV)
        for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
            t.fill_(0x7F)
        st = B.PagedStep(lc, 1, T, DEV, n_pages=kv.n_pages, n_new=ints([T]))
        lay.compact_paged_plan(kv, st)
        q = torch.empty((T, Hq * hd), dtype=dt, device=DEV)
        # (a single row is written by itself: T = 290 and n = 1 is a decode step behind 289 rows)
        cut = T - 1 if n == 1 else T
        for lo, hi in ((0, cut), (cut, T)):
            if lo < hi:
                lay.compact_rope_paged_write(x[lo:hi].reshape(hi - lo, -1).to(DEV), kv, st.slot[lo:hi], st.rot[lo:hi], q[lo:hi])
        cached = kv.rows(0, T)
        assert torch.isfinite(cached[0]).all() and torch.isfinite(cached[1]).all()
        out.append(run_attn(lay, kv, q[T - n:], [n], [T]))
    got = cached[name == "v"][at, 1].cpu()
    if name == "v":
        # half a step of E4M3 is 2^-4 of the value; the top of the range is cut off at 240 * 2^120, less than 2^-4 (1/16) below the largest
        assert ((got[:4] - large[at, Hq + H + 1, :4].float()).abs() <= 2.0 ** -4 * large[at, Hq + H + 1, :4].float().abs()).all()
    before = max(at - (T - n), 0)
    assert torch.equal(out[1][:before], out[0][:before]) and torch.isfinite(out[0]).all()
    if n > 1:
        assert before > 0
    # the other KV head never sees it
    half = Hq // H * hd
    assert torch.equal(out[1][:, :half], out[0][:, :half])


@pytest.mark.parametrize("used", [0, 1, 5])
def test_a_stack_of_2_to_the_31_pages(used):
    """Places on the stack of free pages up to the largest int: pages are taken from its top, and a finished request's are pushed there."""
    lc, n_pages = layer(4, 2, 64), 2 ** 31 - 1
    lay, empty = handle(lc), torch.empty(0, dtype=torch.uint8, device=DEV)
    free = torch.empty(n_pages, dtype=torch.int32, device=DEV)
    n_free = n_pages - used
    free[n_free - 8:] = torch.arange(n_free - 8, n_pages, dtype=torch.int64, device=DEV).int()
    table = ints([[-1] * 8, list(range(100, 100 + used)) + [-1] * (8 - used), [-1] * 8])
    kv = B.PagedKV(lc, empty, empty, empty, empty, table, n_pages=n_pages, page_rows=16)
    st = B.PagedStep(lc, 3, 64, DEV, n_new=ints([33, -1, 0]), len=ints([0, 16 * used, 0]), free=free, n_free=ints([n_free]))
    lay.compact_paged_plan(kv, st)
    stack = list(range(n_free - 8, n_free)) + list(range(100, 100 + used))     # the top of it
    assert kv.table[0].tolist() == stack[:-4:-1] + [-1] * 5
    assert st.n_free_out.item() == n_pages - 3 and st.n_refused.item() == 0 and st.len_out.tolist() == [33, 0, 0]
    # (entries above the new top are not written)
    assert free[n_free - 8:n_pages - 3].tolist() == stack[:-3]
    assert free[n_pages - 3:].tolist() == list(range(n_pages - 3, n_pages))
    assert st.slot[:33].tolist() == [stack[-1 - r // 16] * 16 + r % 16 for r in range(33)] and (st.slot[33:] == -1).all()


def test_arrays_on_the_host_are_refused():
    """One array of a call on the CPU, the others where they belong: nothing is launched."""
    lc = layer(8, 2, 64)
    lay, kv, st = handle(lc), B.PagedKV.allocate(lc, 3, 4, 12, 16, DEV), B.PagedStep(lc, 3, 5, DEV, n_pages=12)
    lay.ensure_paged_workspace(3, 5, 2, 64, DEV)
    qkv, q, o = (torch.zeros((5, n), dtype=torch.bfloat16, device=DEV) for n in (768, 512, 512))

    def calls(qkv=qkv, slot=st.slot, rot=st.rot, q=q, cu=st.cu, kv_len=st.kv_len, o=o, kv=kv):
        lay.compact_rope_paged_write(qkv, kv, slot, rot, q)
        lay.compact_attn_paged(q, kv, cu, kv_len, 2, 64, o)
    lay.compact_paged_plan(kv, st)
    calls()
    for name, t in dict(qkv=qkv, slot=st.slot, rot=st.rot, q=q, cu=st.cu, kv_len=st.kv_len, o=o).items():
        with pytest.raises(B.CompactError) as e:
            calls(**{name: t.cpu()})
        assert e.value.code == 1, name
    for name in ("n_new", "len", "n_free", "free", "n_free_out", "n_refused", "len_out", "kv_len", "cu", "slot", "rot"):
        bad = B.PagedStep(lc, 3, 5, DEV, n_pages=12)
        setattr(bad, name, getattr(bad, name).cpu())
        with pytest.raises(B.CompactError):
            lay.compact_paged_plan(kv, bad)
    for name in ("k", "v", "k_scale", "v_scale", "table"):
        with pytest.raises(B.CompactError):
            B.PagedKV(lc, **{n: getattr(kv, n).cpu() if n == name else getattr(kv, n) for n in ("k", "v", "k_scale", "v_scale", "table")})
    with pytest.raises(B.CompactError):
        calls(kv=B.PagedKV.allocate(lc, 3, 4, 12, 16, "cpu"))
    lay.ws = lay.ws.cpu()
    with pytest.raises(B.CompactError):
        calls()


@pytest.mark.parametrize("lc", [layer(4, 1, 128), layer(2, 1, 64, "fp32")], ids=IDS)
@pytest.mark.parametrize("n_new,lens", [([4000, 1], [5000, 4999]),                                               # by request
                                        ([1, 2, 50] + [1, 0, 3] * 12, [1100, 257, 1090] + [600, 1000, 300] * 12),    # by row
                                        ([1, 1, 1200, 40, 3, 32, 500, 9], [8200, 300, 6000, 8200, 8200, 4100, 7000, 513])],   # by both
                         ids=["by_request", "by_row", "by_both"])
def test_records_stay_inside_the_workspace_that_was_asked_for(lc, n_new, lens):
    """Every way to lay out the records of split keys, in a workspace of that size: right, the bits of the requests by themselves, and
    what lies behind it is untouched."""
    kv, ref, table = random_cache(lc, lens, 64, 23)
    q, lay = queries(lc, sum(n_new), 23), handle(lc)
    said = [L if n else 0 for n, L in zip(n_new, lens)]
    need = lay.paged_workspace_bytes(len(lens), sum(n_new), max(n_new), max(lens))
    room = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    lay.ws = room[:need]
    o = run_attn(lay, kv, q, n_new, said)
    assert lay.ws.data_ptr() == room.data_ptr() and (room[need:] == 0xA5).all()
    check_attn(lc, q, o, n_new, said, ref, table)
    lay.ws, row = None, 0
    for i, (n, L) in enumerate(zip(n_new, said)):
        if n:
            one = B.PagedKV(lc, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.table[i:i + 1].contiguous())
            assert torch.equal(run_attn(lay, one, q[row:row + n], [n], [L]), o[row:row + n]), i
        row += n
